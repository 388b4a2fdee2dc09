"""GPU: flashmask_decode_tree and flashmask_cache_accept against their definitions.  Wherever nothing is cached, and in keys that no row of a call sees,
the pages hold NaN and infinities."""
import numpy as np
import pytest
import torch

from keys_util import ints, paged, queries, values_of
from oracle import cache_oracle, keys_oracle as orc
from serving_util import check, decode_bounds, f64, raw

pytestmark = pytest.mark.gpu


def _parents(kind, B, T, seed):
    rng = np.random.default_rng(seed)
    at = np.arange(T)
    if kind == "chain":
        return np.tile(at - 1, (B, 1))
    if kind == "star":
        return np.full((B, T), -1)
    if kind == "odd":           # numbers that name no token ahead: such a token follows the sequence
        p = rng.integers(-3, T + 3, (B, T))
        p[:, ::4] = rng.choice([1 << 30, -(1 << 31), T], p[:, ::4].shape)
        return p
    return np.where(rng.random((B, T)) < 0.2, -1, at - rng.integers(1, 9, (B, T))).clip(-1)


def _problem(seed, lens, H, Hk, T, d, page, type, cache, packed=False, columns=None, mask="none", holes=(), kind="tree"):
    p = paged(seed, lens, Hk, page, d, cache, packed, columns, holes)
    rng = np.random.default_rng(seed)
    lens, N, B = np.array(lens), p["table"].shape[1] * page, len(lens)
    p["window"], bounds = {"window": 37, "narrow": 3}.get(mask, 0), None
    if mask == "bounds":
        n = max(N - page // 2, 1)
        lts = np.full((B, n), N)
        for b, L in enumerate(lens):
            lts[b, L // 3:L // 2], lts[b, L // 2:L * 3 // 4] = L // 2, L * 3 // 4
        lte, uts, ute = np.full_like(lts, N), np.zeros_like(lts), np.zeros_like(lts)
        uts[:, ::3], ute[:, ::3] = lens[:, None] - T, lens[:, None] - T + 2     # from the tokens of the first two generations
        bounds = (lts, lte, uts, ute)
    elif mask == "random":
        bounds = rng.integers(-2, N + 3, (4, B, N))
    parents = _parents(kind, B, T, seed)
    table = p["table"].cpu().numpy()
    for b, L in enumerate(lens):
        lines, mine = orc.ancestors(parents[b]), None if bounds is None else [x[b] for x in bounds]
        for j in range(min(L, N)):
            at = cache_oracle.place(table, len(p["k_cache"]), page, b, j)
            if at is not None and not any(orc.tree_visible(L, T, lines, t, j, p["window"], mine) for t in range(T)):
                p["k_cache"][at[0], :, at[1]] = p["v_cache"][at[0], :, at[1]] = torch.nan
    return p | {"q": queries(seed, B, H, T, d, type, packed), "scale": d ** -0.5, "parents": parents, "np_bounds": bounds}


def _call(p, **more):
    import paper_2410_01359_amd as fm
    bounds = None if p["np_bounds"] is None else tuple(ints(x) for x in p["np_bounds"])
    return fm.flashmask_decode_tree(p["q"], p["k_cache"], p["v_cache"], p["table"], p["lens"], ints(p["parents"]), p["scale"], bounds=bounds,
                                    window=p["window"], k_scale=p["k_scale"], v_scale=p["v_scale"], **more)


def _check(p, type, what=""):
    out, lse = _call(p)
    k, v = values_of(p)
    ref, ref_lse, mass, size = orc.decode_tree(f64(p["q"]), k, v, p["table"].cpu().numpy(), p["lens"].cpu().numpy(), p["parents"], p["scale"],
                                               p["window"], p["np_bounds"])
    assert out.dtype == p["q"].dtype and out.shape == p["q"].shape and lse.dtype == torch.float32
    bound, lse_bound = decode_bounds(type, ref, ref_lse, mass, size, ref.shape[-1], max(int(p["lens"].max()), 1))
    got_lse = f64(lse)
    assert np.array_equal(np.isneginf(got_lse), np.isneginf(ref_lse)), f"{what}: rows without keys differ"
    assert (f64(out)[np.isneginf(ref_lse)] == 0).all()
    some = ~np.isneginf(ref_lse)
    check(f64(out), ref, bound, what + "out")
    check(got_lse[some], ref_lse[some], lse_bound[some], what + "lse")


CASES = [
    # lens, H, Hk, T, d, page, columns
    ([1], 1, 1, 1, 64, 16, None),
    ([2, 9, 0, 17, 31, 33], 4, 4, 3, 128, 16, None),
    ([5, 0, 130, 64, 333], 8, 8, 7, 128, 64, None),
    ([333, 7], 5, 1, 9, 64, 48, None),                      # 45 query rows to a K/V head
    ([30, 100, 1, 257], 8, 2, 16, 64, 32, None),            # 64 rows, sequences shorter than the tree
    ([129, 64], 12, 1, 26, 128, 16, None),                  # 312 rows
    ([300, 90], 4, 1, 64, 64, 256, None),
    ([700, 40], 2, 1, 130, 128, 16, None),                  # trees of several words
    ([300], 2, 2, 256, 64, 16, 24),                         # the largest tree, rows of the table beyond what is used
    ([1025, 40, 0, 2111, 1], 8, 2, 5, 128, 64, None),       # split
    ([2500, 1500], 16, 2, 12, 64, 128, None),
]


@pytest.mark.parametrize("type,cache", [("bf16", "bf16"), ("f16", "f16"), ("bf16", "e4m3"), ("f16", "e4m3")])
@pytest.mark.parametrize("case", range(len(CASES)))
def test_against_the_definition(case, type, cache):
    lens, H, Hk, T, d, page, columns = CASES[case]
    _check(_problem(case, lens, H, Hk, T, d, page, type, cache, packed=case % 2 == 1, columns=columns), type)


@pytest.mark.parametrize("type,cache", [("bf16", "bf16"), ("f16", "e4m3")])
@pytest.mark.parametrize("mask", ["window", "narrow", "bounds", "random"])
@pytest.mark.parametrize("case", [1, 2, 3, 4, 5, 7, 9, 10])
def test_masks(case, mask, type, cache):
    lens, H, Hk, T, d, page, columns = CASES[case]
    _check(_problem(100 + case, lens, H, Hk, T, d, page, type, cache, packed=case % 2 == 0, columns=columns, mask=mask), type)


@pytest.mark.parametrize("kind", ["chain", "star", "odd"])
@pytest.mark.parametrize("case", [1, 2, 4, 5, 6, 7])
def test_shapes_of_trees(case, kind):
    lens, H, Hk, T, d, page, columns = CASES[case]
    _check(_problem(200 + case, lens, H, Hk, T, d, page, "bf16", "bf16", columns=columns, kind=kind), "bf16")


def test_pages_that_are_missing():
    _check(_problem(5, [100, 40, 64], 8, 2, 12, 64, 16, "bf16", "bf16", holes=((0, 1, -1), (0, 6, 10 ** 6), (1, 2, -7), (2, 0, -1))), "bf16")


@pytest.mark.parametrize("T,H,Hk", [(6, 4, 4), (40, 8, 2)])
@pytest.mark.parametrize("type,odd", [("bf16", torch.inf), ("f16", -torch.inf), ("bf16", torch.nan)])
def test_an_odd_value_reaches_those_that_see_it(type, odd, T, H, Hk):
    """An infinite or NaN value of a drafted token's key: its descendants and itself have it, nobody else does."""
    p = _problem(6, [70], H, Hk, T, 64, 16, type, type)
    start, u = 70 - T, 2
    at = cache_oracle.place(p["table"].cpu().numpy(), len(p["v_cache"]), 16, 0, start + u)
    p["v_cache"][at[0], :, at[1], 5] = odd
    lines = orc.ancestors(p["parents"][0])
    out = f64(_call(p)[0])[0]
    for t in range(T):
        hit = out[:, t, 5]
        if u in lines[t]:
            assert (np.isnan(hit) if np.isnan(odd) else hit == odd).all(), t
        else:
            assert np.isfinite(hit).all(), t
        assert np.isfinite(np.delete(out[:, t], 5, -1)).all()


MORE_CASES = [
    # more sequences than a wave looks over at once; with that many workgroups the chunks of keys are listed by a launch of their own
    ([(37 * b) % 150 for b in range(70)], 16, 16, 64, 64, 16),
    ([(37 * b) % 150 for b in range(130)], 4, 2, 9, 64, 16),
    ([(91 * b) % 700 for b in range(70)], 2, 1, 40, 128, 32),
    # few chunks to a sequence, and many rows: a join of their own
    ([1500, 700, 20, 0], 32, 16, 40, 64, 32),
    ([2200, 900], 16, 4, 61, 128, 64),
]


@pytest.mark.parametrize("mask", ["none", "window", "bounds"])
@pytest.mark.parametrize("case", range(len(MORE_CASES)))
def test_many_sequences_and_heads(case, mask):
    lens, H, Hk, T, d, page = MORE_CASES[case]
    _check(_problem(300 + case, lens, H, Hk, T, d, page, ("bf16", "f16")[case % 2], ("e4m3", "f16", "bf16", "f16", "bf16")[case], mask=mask),
           ("bf16", "f16")[case % 2])


NARROW_CASES = [
    # few rows to a K/V head, many tokens
    ([700, 90, 61, 0], 4, 4, 60, 64, 16),
    ([300, 63, 20], 3, 3, 63, 128, 32),
    ([130, 40, 1], 2, 2, 33, 64, 48),
    ([2100], 2, 1, 31, 128, 16),
]


@pytest.mark.parametrize("type,cache", [("bf16", "bf16"), ("f16", "e4m3")])
@pytest.mark.parametrize("mask,kind", [("none", "random"), ("none", "chain"), ("none", "star"), ("window", "random"), ("narrow", "chain"), ("bounds", "random"),
                                       ("random", "random"), ("none", "odd")])
@pytest.mark.parametrize("case", range(len(NARROW_CASES)))
def test_many_tokens_of_few_rows(case, mask, kind, type, cache):
    lens, H, Hk, T, d, page = NARROW_CASES[case]
    _check(_problem(500 + case, lens, H, Hk, T, d, page, type, cache, mask=mask, kind=kind), type)


def test_two_graphs_at_once():
    """Calls with workspaces of their own, captured and replayed on two streams at a time, give what each gives alone."""
    import paper_2410_01359_amd as fm
    problems = [_problem(400 + i, [2000, 700, 40], 8, 2, T, 64, 16, "bf16", "bf16") for i, T in enumerate((20, 40))]
    graphs, results, wants, spaces = [], [], [], []     # a graph's workspace lives as long as it does
    for p in problems:
        p["parents_on_gpu"] = ints(p["parents"])
        spaces.append(torch.empty(fm.flashmask_decode_tree_workspace_bytes(3, 8, 2, p["q"].shape[2], 64), dtype=torch.uint8, device="cuda"))

        def call(p=p, ws=spaces[-1]):
            return fm.flashmask_decode_tree(p["q"], p["k_cache"], p["v_cache"], p["table"], p["lens"], p["parents_on_gpu"], p["scale"], workspace=ws)

        wants.append([x.clone() for x in call()])
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=torch.cuda.Stream()):
            results.append(call())
        graphs.append(graph)
    streams = [torch.cuda.Stream() for _ in graphs]
    for _ in range(3):
        for got in results:
            for x in got:
                x.fill_(-7)
        torch.cuda.synchronize()
        for graph, stream in zip(graphs, streams):
            with torch.cuda.stream(stream):
                graph.replay()
        torch.cuda.synchronize()
        for got, want in zip(results, wants):
            assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_a_chain_is_flashmask_decode():
    import paper_2410_01359_amd as fm
    p = _problem(7, [900, 33], 4, 2, 4, 128, 16, "bf16", "bf16", kind="chain")
    want = fm.flashmask_decode(p["q"], p["k_cache"], p["v_cache"], p["table"], p["lens"], p["scale"])
    for a, b in zip(_call(p), want):
        assert torch.allclose(a.float(), b.float(), atol=2.0 ** -7)


def test_on_a_stream_of_its_own_and_in_a_graph():
    import paper_2410_01359_amd as fm
    p = _problem(8, [2000, 700, 40], 8, 2, 20, 64, 16, "bf16", "bf16")
    p["parents"] = ints(p["parents"])
    ws = torch.empty(fm.flashmask_decode_tree_workspace_bytes(3, 8, 2, 20, 64), dtype=torch.uint8, device="cuda")

    def call():
        return fm.flashmask_decode_tree(p["q"], p["k_cache"], p["v_cache"], p["table"], p["lens"], p["parents"], p["scale"], workspace=ws)

    want = [x.clone() for x in call()]
    torch.cuda.synchronize()
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        got = call()
    for _ in range(3):
        for x in got:
            x.fill_(-7)
        ws.fill_(255)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want))


# --- accept
def _paths(B, T, P, seed):
    rng = np.random.default_rng(seed)
    out = np.full((B, P), -1)
    for b in range(B):
        n = int(rng.integers(0, min(P, T) + 1))
        out[b, :n] = np.sort(rng.choice(T, n, replace=False))
    return out


def _accept(p, pools, T, paths):
    import paper_2410_01359_amd as fm
    table, lens = p["table"].cpu().numpy(), p["lens"].cpu().numpy()
    want, want_lens = orc.accept([f64(x) for x in pools], table, lens, T, paths)
    got = fm.flashmask_cache_accept(pools, p["table"], p["lens"], T, ints(paths))
    assert np.array_equal(got.cpu().numpy(), want_lens)
    for i, (a, b) in enumerate(zip(pools, want)):
        assert np.array_equal(f64(a), b, equal_nan=True), i


@pytest.mark.parametrize("cache", ["bf16", "f16", "e4m3"])
@pytest.mark.parametrize("lens,heads,T,P,d,page", [
    ([1], 1, 1, 1, 64, 16), ([40, 3, 0, 17, 200], 2, 5, 4, 128, 16), ([70, 64, 130], 8, 20, 20, 64, 32), ([300, 256, 299], 3, 256, 256, 128, 48),
    ([33, 100] * 9, 20, 12, 9, 64, 16)])
def test_accept(lens, heads, T, P, d, page, cache):
    p = paged(T, lens, heads, page, d, cache, packed=T % 2 == 0, junk=cache != "e4m3")
    _accept(p, [p["k_cache"], p["v_cache"]], T, _paths(len(lens), T, P, T))


def test_accept_many_pools():
    p = paged(50, [60, 44], 2, 16, 64, "bf16")
    gen = torch.Generator(device="cuda").manual_seed(1)
    pools = [torch.randn(p["k_cache"].shape, device="cuda", generator=gen).bfloat16() for _ in range(70)]
    _accept(p, pools, 9, np.array([[0, 2, 3, 4, 8], [5, 6, -1, -1, -1]]))


def test_accept_odd_paths_and_missing_pages():
    """A path ends in front of what is no drafted token or does not ascend; from a place without a page come zeros, and to one goes nothing."""
    p = paged(51, [60, 60, 60, 60, 90], 2, 16, 64, "bf16", holes=((3, 3, -1), (0, 3, -1)))
    p["lens"] = ints([60, 60, 60, 60, 70])       # the last ends behind the table
    paths = np.array([[1, 14, 15, -1], [3, 3, 5, 6], [2, 16, 3, 4], [0, 4, 13, 14], [0, 5, 8, 15]])
    _accept(p, [p["k_cache"], p["v_cache"]], 16, paths)


def test_accept_a_pool_named_twice_is_refused():
    import paper_2410_01359_amd as fm
    p = paged(3, [40], 2, 16, 64, "bf16")
    before = p["k_cache"].clone()
    with pytest.raises(fm.FlashMaskError):
        fm.flashmask_cache_accept([p["k_cache"], p["v_cache"], p["k_cache"]], p["table"], p["lens"], 5, ints([[1, 2]]))
    assert torch.equal(raw(before), raw(p["k_cache"]))


def test_accept_pools_of_another_layout_are_refused():
    import paper_2410_01359_amd as fm
    p = paged(3, [40], 2, 16, 64, "bf16")
    k, other = p["k_cache"], torch.zeros_like(p["k_cache"].transpose(1, 2).contiguous()).transpose(1, 2)
    for pools in ([k, other], [other, k], [k, other.float()], [k, other[1:]]):
        with pytest.raises(fm.FlashMaskError):
            fm.flashmask_cache_accept(pools, p["table"], p["lens"], 5, ints([[1, 2]]))
    fm.flashmask_cache_accept([other, torch.zeros_like(other)], p["table"], p["lens"], 5, ints([[1, 2]]))
    torch.cuda.synchronize()


def test_accept_a_graph_of_it():
    import paper_2410_01359_amd as fm
    p = paged(52, [60, 44], 2, 16, 64, "bf16")
    path = ints([[3, 4], [1, 8]])
    start = [raw(p[n]).clone() for n in ("k_cache", "v_cache")]
    fm.flashmask_cache_accept([p["k_cache"], p["v_cache"]], p["table"], p["lens"], 9, path)
    want = [raw(p[n]).clone() for n in ("k_cache", "v_cache")]
    torch.cuda.synchronize()
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        lens = fm.flashmask_cache_accept([p["k_cache"], p["v_cache"]], p["table"], p["lens"], 9, path)
    for _ in range(3):
        for n, x in zip(("k_cache", "v_cache"), start):
            raw(p[n]).copy_(x)
        lens.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert lens.tolist() == [53, 37]
        assert all(torch.equal(raw(p[n]), x) for n, x in zip(("k_cache", "v_cache"), want))
