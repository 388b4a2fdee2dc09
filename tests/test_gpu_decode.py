"""GPU: flashmask_decode against the definition in 64 bits.  Wherever nothing is cached (the rest of last pages, pages of nobody) and in
keys that no row of the call sees the caches hold NaN and infinities."""
import numpy as np
import pytest
import torch

from serving_util import TYPES, cache_of, check, decode_bounds, f64, orc, raw, rounding, rows_of, strided

pytestmark = pytest.mark.gpu


def _ints(x):
    return torch.tensor(np.asarray(x), dtype=torch.int32, device="cuda")


def _problem(seed, lens, H, Hk, T, d, page, type, cache, packed=False, columns=None, mask="none", holes=()):
    """Arguments of flashmask_decode by name; holes: (sequence, column, entry) of the table that name no page."""
    rng = np.random.default_rng(seed)
    gen = torch.Generator(device="cuda").manual_seed(seed)
    lens = np.array(lens)
    B, counts = len(lens), -(-lens // page)
    columns = columns or max(1, counts.max())
    counts = np.minimum(counts, columns)
    num_pages = int(counts.sum()) + 3
    order, table = rng.permutation(num_pages), np.full((B, columns), -1, np.int64)
    for b, n in enumerate(counts):
        table[b, :n] = order[counts[:b].sum():counts[:b].sum() + n]
    for b, c, entry in holes:
        table[b, c] = entry
    window, bounds = 0, None
    N = columns * page
    if mask == "window":
        window = 37
    elif mask == "bounds":      # questions with answers that do not see each other, an interval that hides every third key, short vectors
        columns_of = max(N - page // 2, 1)
        lts = np.full((B, columns_of), N)
        for b, n in enumerate(lens):
            lts[b, n // 3:n // 2], lts[b, n // 2:n * 3 // 4] = n // 2, n * 3 // 4
        lte = np.full_like(lts, N)
        uts, ute = np.zeros_like(lts), np.zeros_like(lts)
        uts[:, ::3], ute[:, ::3] = lens[:, None] - T, lens[:, None] - T + (T + 1) // 2      # from the first half of the new rows
        bounds = (lts, lte, uts, ute)
    caches = []
    for _ in range(2):
        c = cache_of(gen, cache, num_pages, Hk, page, d, packed, junk=True)
        at = rows_of(c, table, lens)
        if at is not None:
            raw(c)[at[0], :, at[1]] = raw(cache_of(gen, cache, len(at[0]), Hk, 16, d)[:, :, 0].contiguous())
        for b, n in enumerate(lens):
            for j in range(min(n, N)):
                if 0 <= table[b, j // page] < num_pages and not any(orc.visible(n, t, T, j, window, None if bounds is None else [x[b] for x in bounds]) for t in range(T)):
                    c[table[b, j // page], :, j % page] = torch.nan
        caches.append(c)
    scales = [torch.rand(Hk, device="cuda", generator=gen) + 0.5 for _ in range(2)] if cache == "e4m3" else [None, None]
    q = torch.randn((B, T, H, d) if packed else (B, H, T, d), device="cuda", generator=gen).to(TYPES[type])
    return {"q": q.transpose(1, 2) if packed else q, "k_cache": caches[0], "v_cache": caches[1], "table": _ints(table), "lens": _ints(lens),
            "scale": d ** -0.5, "window": window, "bounds": None if bounds is None else tuple(_ints(x) for x in bounds),
            "k_scale": scales[0], "v_scale": scales[1]}


def _reference(a):
    k, v = f64(a["k_cache"]), f64(a["v_cache"])
    if a["k_scale"] is not None:
        k, v = (x * f64(s)[:, None, None] for x, s in ((k, a["k_scale"]), (v, a["v_scale"])))
    bounds = None if a["bounds"] is None else [x.cpu().numpy() for x in a["bounds"]]
    return orc.decode(f64(a["q"]), k, v, a["table"].cpu().numpy(), a["lens"].cpu().numpy(), a["scale"], a["window"], bounds)


def _check(a, type, got=None, what=""):
    import paper_2410_01359_amd as fm
    out, lse = got or fm.flashmask_decode(**a)
    ref, ref_lse, mass, size = _reference(a)
    assert out.dtype == a["q"].dtype and out.shape == a["q"].shape and lse.dtype == torch.float32
    bound, lse_bound = decode_bounds(type, ref, ref_lse, mass, size, ref.shape[-1], int(a["lens"].max()))
    got_lse = f64(lse)
    assert np.array_equal(np.isneginf(got_lse), np.isneginf(ref_lse)), f"{what}: rows without keys differ"
    assert (f64(out)[np.isneginf(ref_lse)] == 0).all()
    some = ~np.isneginf(ref_lse)
    check(f64(out), ref, bound, what + "out")
    check(got_lse[some], ref_lse[some], lse_bound[some], what + "lse")


CASES = [
    # lens, H, Hk, T, d, page, columns
    ([1], 1, 1, 1, 64, 16, None),
    ([0, 1, 2, 15, 16, 17, 31, 33], 4, 4, 1, 128, 16, None),
    ([5, 0, 130, 64, 333], 8, 8, 1, 128, 64, None),
    ([333, 7], 5, 1, 1, 64, 48, None),
    ([3, 100, 1, 0, 257], 8, 2, 4, 64, 32, None),          # sequences shorter than the new tokens
    ([129, 64], 40, 5, 5, 128, 16, None),                  # 40 query rows to a K/V head
    ([300, 9], 16, 2, 8, 128, 256, None),                  # 64 rows
    ([70, 200], 32, 2, 5, 64, 16, None),                   # 80 rows: two blocks
    ([1025, 40, 0, 2111, 1], 8, 2, 1, 128, 64, None),      # split
    ([3000], 4, 4, 2, 64, 16, None),
    ([700, 2500, 3, 1500], 24, 3, 3, 128, 48, 70),         # rows of the table beyond what is used
    ([2000, 2048, 1999], 16, 2, 8, 64, 128, None),
]


@pytest.mark.parametrize("type,cache", [("bf16", "bf16"), ("f16", "f16"), ("bf16", "e4m3"), ("f16", "e4m3")])
@pytest.mark.parametrize("case", range(len(CASES)))
def test_against_the_definition(case, type, cache):
    lens, H, Hk, T, d, page, columns = CASES[case]
    _check(_problem(case, lens, H, Hk, T, d, page, type, cache, packed=case % 2 == 1, columns=columns), type)


@pytest.mark.parametrize("type,cache", [("bf16", "bf16"), ("f16", "e4m3")])
@pytest.mark.parametrize("mask", ["window", "bounds"])
@pytest.mark.parametrize("case", [1, 2, 4, 5, 7, 8, 10, 11])
def test_masks(case, mask, type, cache):
    lens, H, Hk, T, d, page, columns = CASES[case]
    _check(_problem(100 + case, lens, H, Hk, T, d, page, type, cache, packed=case % 2 == 0, columns=columns, mask=mask), type)


@pytest.mark.parametrize("type,cache", [("bf16", "bf16"), ("f16", "e4m3")])
@pytest.mark.parametrize("mask", ["none", "window"])
@pytest.mark.parametrize("B,long", [(65, 1300), (130, 1100), (64, 2000)])
def test_more_sequences_than_lanes(B, long, mask, type, cache):
    """Lengths are added up 64 sequences at a time: the longest on either side of a round."""
    rng = np.random.default_rng(B)
    lens = rng.integers(0, 40, size=B)
    lens[[0, 63, B - 1]] = long, long - 77, long - 1
    _check(_problem(200 + B, lens, 4, 2, 1, 64, 16, type, cache, mask=mask), type)


@pytest.mark.parametrize("mask", ["none", "bounds"])
@pytest.mark.parametrize("lens,H,Hk,T,d,packed", [([90, 300, 20], 2, 1, 70, 64, False), ([1500, 260], 3, 3, 40, 128, True), ([400], 2, 2, 256, 64, False)])
def test_many_new_tokens(lens, H, Hk, T, d, packed, mask):
    """Several blocks of query rows to a K/V head, an odd number of them among two teams of waves."""
    _check(_problem(300 + T, lens, H, Hk, T, d, 16, "bf16", "bf16", packed=packed, mask=mask), "bf16")


@pytest.mark.parametrize("type,cache,d", [("bf16", "bf16", 64), ("f16", "e4m3", 64), ("bf16", "e4m3", 128)])
@pytest.mark.parametrize("H,Hk", [(3, 3), (10, 5), (40, 1), (66, 3)])
def test_odd_numbers_of_heads_side_by_side(H, Hk, type, cache, d):
    _check(_problem(400 + H, [700, 1090, 5], H, Hk, 1, d, 32, type, cache, packed=True), type)


@pytest.mark.parametrize("mask", ["none", "bounds"])
def test_pages_that_are_none(mask):
    """Holes in the table, and lengths beyond it: keys without a page are not seen."""
    big = np.iinfo(np.int32).max
    holes = ((0, 1, -1), (0, 3, 1000), (1, 0, big), (1, 1, -big - 1), (2, 0, -7))
    a = _problem(7, [100, 40, 10, 5000], 4, 2, 2, 64, 16, "bf16", "bf16", columns=7, mask=mask, holes=holes)
    _check(a, "bf16", what="whole ")
    a = _problem(8, [1500, 1030, 10, big], 4, 2, 1, 128, 16, "f16", "f16", columns=100, mask=mask, holes=holes)
    _check(a, "f16", what="split ")
    a["lens"] = _ints([-1, -big - 1, 0, -16])
    _check(a, "f16", what="negative lengths ")


@pytest.mark.parametrize("mask", [None, "window", "bounds"])
@pytest.mark.parametrize("type,cache", [("bf16", "bf16"), ("f16", "e4m3")])
@pytest.mark.parametrize("lens", [[70, 90], [1100, 1470]])
def test_odd_values_that_some_rows_see(lens, type, cache, mask):
    """NaN and infinities among the values of keys that some new rows see and others do not reach those rows alone."""
    import paper_2410_01359_amd as fm
    T, H, Hk, d, page = 4, 12, 2, 128, 16
    a = _problem(9, lens, H, Hk, T, d, page, type, "f16" if cache == "f16" else cache)
    table = a["table"].cpu().numpy()
    if mask == "window":
        a["window"] = 20
    elif mask == "bounds":
        N = table.shape[1] * page
        lts = np.full((2, N), N)
        lts[:, 30:34] = np.array(lens)[:, None] - 2         # hidden from the last two rows
        a["bounds"] = tuple(_ints(x) for x in (lts, np.full((2, N), N), np.zeros((2, N)), np.zeros((2, N))))
    clean, clean_lse = fm.flashmask_decode(**a)
    ref, _, _, _ = _reference(a)
    for b, n in enumerate(lens):
        at = {None: [n - 1, n - 3], "window": [n - 1, n - 22], "bounds": [31, n - 2]}[mask]
        for j, odd in zip(at, (torch.nan, torch.nan if cache == "e4m3" else -torch.inf)):
            a["v_cache"][table[b, j // page], :, j % page, 5] = odd
        bounds = None if a["bounds"] is None else [x[b].cpu().numpy() for x in a["bounds"]]
        for t in range(T):
            ref[b, :, t, 5] += sum(float("nan") if k == 0 or cache == "e4m3" else float("-inf") for k, j in enumerate(at)
                                   if orc.visible(n, t, T, j, a["window"], bounds))
    out, lse = fm.flashmask_decode(**a)
    assert torch.equal(lse, clean_lse)
    got, odd = f64(out), ~np.isfinite(ref)
    assert odd.any() and not odd[..., :5].any()
    assert np.array_equal(np.isnan(got), np.isnan(ref)) and np.array_equal(np.isneginf(got), np.isneginf(ref))
    off = np.abs(got - f64(clean))[~odd]
    assert (off <= 2 * rounding(type, f64(clean))[~odd] + 2.0 ** -20).all()


def test_every_8_bit_value():
    """A sequence of one token returns its values."""
    import paper_2410_01359_amd as fm
    codes = torch.arange(256, dtype=torch.uint8)
    codes[127] = codes[255] = 0     # NaN
    cache = codes.view(2, 1, 1, 128).expand(2, 1, 16, 128).contiguous().cuda().view(torch.float8_e4m3fn)
    one = torch.ones(1, device="cuda")
    for type in (torch.bfloat16, torch.float16):
        q = torch.zeros((2, 1, 1, 128), device="cuda", dtype=type)
        out, lse = fm.flashmask_decode(q, cache, cache, _ints([[0], [1]]), _ints([1, 1]), 1.0, k_scale=one, v_scale=one)
        assert torch.equal(out.float(), cache[:, :, :1].float()) and (lse == 0).all()
        # and as keys: with a query of one element set, lse is that element
        for at in range(0, 128, 7):
            q = torch.zeros((2, 1, 1, 128), device="cuda", dtype=type)
            q[..., at] = 1
            _, lse = fm.flashmask_decode(q, cache, cache, _ints([[0], [1]]), _ints([1, 1]), 1.0, k_scale=one, v_scale=one)
            want = cache[:, 0, 0, at].float()
            assert ((lse[:, 0, 0] - want).abs() <= 2.0 ** -22 * want.abs()).all()


def test_odd_queries_and_keys_reach_their_own_rows():
    import paper_2410_01359_amd as fm
    a = _problem(11, [200, 50], 8, 2, 2, 64, 16, "bf16", "bf16")
    clean, _ = fm.flashmask_decode(**a)
    a["q"][0, 5, 1, 3] = torch.nan
    out, lse = fm.flashmask_decode(**a)
    assert out[0, 5, 1].isnan().all() and lse[0, 5, 1].isnan()
    out[0, 5, 1] = clean[0, 5, 1]
    assert torch.equal(out, clean)
    a = _problem(11, [200, 50], 8, 2, 2, 64, 16, "bf16", "bf16")
    a["k_cache"][a["table"][1, 3].item(), 0, 0, 0] = torch.nan    # key 48, which both rows of sequence 1 see
    out, _ = fm.flashmask_decode(**a)
    assert out[1, :4].isnan().all()
    out[1, :4] = clean[1, :4]
    assert torch.equal(out, clean)


def test_large_scores():
    """Scores of thousands: the running maximum, and rows whose weight lies in one key."""
    a = _problem(12, [1500, 600], 4, 2, 2, 128, 32, "bf16", "bf16")
    a["scale"] = 60.0
    _check(a, "bf16")


def test_long_sequence():
    a = _problem(13, [40007], 2, 1, 1, 64, 256, "bf16", "bf16")
    _check(a, "bf16")


def test_offsets_beyond_32_bits():
    """Pages on either side of 4 GiB and of 2^31 elements."""
    import paper_2410_01359_amd as fm
    num_pages, page, d = 1 << 21, 16, 128                    # 8 GiB each
    caches = [torch.empty((num_pages, 1, page, d), device="cuda", dtype=torch.bfloat16) for _ in range(2)]
    pages = [3, (1 << 20) - 1, 1 << 20, (1 << 20) + 1, num_pages - 1]
    gen = torch.Generator(device="cuda").manual_seed(3)
    small = [torch.randn((len(pages), 1, page, d), device="cuda", generator=gen).bfloat16() for _ in range(2)]
    for c, s in zip(caches, small):
        c[torch.tensor(pages, device="cuda")] = s
    q = torch.randn((1, 2, 1, d), device="cuda", generator=gen).bfloat16()
    got = fm.flashmask_decode(q, *caches, _ints([pages]), _ints([77]), 0.1)
    want = fm.flashmask_decode(q, *small, _ints([range(len(pages))]), _ints([77]), 0.1)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    token = torch.randn((1, 1, d), device="cuda", generator=gen).bfloat16()
    fm.flashmask_cache_append(token, token, *caches, _ints([pages]), _ints([0]), _ints([79]))
    assert torch.equal(caches[0][-1, :, 15], token[0]) and torch.equal(caches[1][-1, :, 15], token[0])
    fm.flashmask_cache_fork(caches, _ints([pages]), _ints([70]), _ints([0]), _ints([(1 << 20) + 5]), page)
    for c in caches:
        assert torch.equal(c[(1 << 20) + 5], c[-1])


def test_same_bits_whatever_the_workspace_holds():
    import paper_2410_01359_amd as fm
    a = _problem(14, [2000, 1100, 0, 300], 16, 4, 2, 128, 16, "bf16", "e4m3")
    need = fm.flashmask_decode_workspace_bytes(4, 16, 4, 2, 128)
    ws = torch.full((need,), 255, dtype=torch.uint8, device="cuda")
    first = fm.flashmask_decode(**a, workspace=ws)
    for fill in (0, 127, None):
        if fill is not None:
            ws.fill_(fill)
        again = fm.flashmask_decode(**a, workspace=ws if fill is not None else None)
        assert torch.equal(first[0], again[0]) and torch.equal(first[1], again[1])
    with pytest.raises(fm.FlashMaskError):
        fm.flashmask_decode(**a, workspace=ws[:need - 256])


def test_refusals():
    import paper_2410_01359_amd as fm
    a = _problem(15, [20, 30], 4, 2, 1, 64, 16, "bf16", "bf16")
    fm.flashmask_decode(**a)
    q, table, lens, cache = a["q"], a["table"], a["lens"], a["k_cache"]
    vec = torch.zeros((2, 32), dtype=torch.int32, device="cuda")
    for wrong in ({"q": q.half()}, {"q": q.float()}, {"q": q[:1]}, {"q": q[:, :3]}, {"q": q[..., :32]}, {"q": q.cpu()}, {"q": q[:, :, :0]}, {"q": q[:, 0]},
                  {"lens": lens[:1]}, {"lens": lens.long()}, {"lens": lens.cpu()}, {"table": table[:1]}, {"table": table[:, :0]}, {"scale": 0.0},
                  {"scale": float("nan")}, {"window": -1}, {"bounds": (vec,) * 3}, {"bounds": (vec,) * 3 + (vec[:1],)}, {"bounds": (vec[:, :0],) * 4},
                  {"bounds": (vec.long(),) * 4}, {"k_scale": torch.ones(2, device="cuda")}, {"k_cache": cache[:, :, :8], "v_cache": cache[:, :, :8]},
                  {"workspace": torch.empty(8, dtype=torch.uint8, device="cuda")}):
        with pytest.raises(fm.FlashMaskError):
            fm.flashmask_decode(**(a | wrong))
    torch.cuda.synchronize()


@pytest.mark.parametrize("lens", [[333, 20], [1500, 700]])
def test_graph_replays_a_decoding_step(lens):
    """Append, decode and fork recorded into a graph, replayed with eager work in between, against eager calls."""
    import paper_2410_01359_amd as fm
    a = _problem(16, lens, 8, 2, 1, 128, 16, "bf16", "bf16", columns=100)
    gen = torch.Generator(device="cuda").manual_seed(4)
    freqs = 10000.0 ** (-torch.arange(64, device="cuda", dtype=torch.float64) / 64)
    qkv = torch.randn((2, 12, 128), device="cuda", generator=gen).bfloat16()
    seqs, at, parents, new = _ints([0, 1]), a["lens"] - 1, _ints([1, 0]), _ints([-1, -1])
    ws = torch.empty(fm.flashmask_decode_workspace_bytes(2, 8, 2, 1, 128), dtype=torch.uint8, device="cuda")
    plan = torch.empty(fm.flashmask_cache_plan_bytes(a["k_cache"].shape[0]), dtype=torch.uint8, device="cuda")
    pools = [a["k_cache"], a["v_cache"]]

    def step():
        q = fm.flashmask_cache_append(qkv[:, 8:10], qkv[:, 10:], *pools, a["table"], seqs, at, q=qkv[:, :8], freqs=freqs)
        out = fm.flashmask_decode(**(a | {"q": q[:, :, None]}), workspace=ws)
        return (*out, *fm.flashmask_cache_fork(pools, a["table"], a["lens"], parents, new, 16),
                *fm.flashmask_cache_free_list(a["table"], pools[0].shape[0], workspace=plan))

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = step()
    for trial in range(4):
        qkv.copy_(torch.randn(qkv.shape, device="cuda", generator=gen).bfloat16())
        eager = [x.clone() for x in step()]
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for x, y in zip(eager, captured):
            assert torch.equal(x, y), trial
