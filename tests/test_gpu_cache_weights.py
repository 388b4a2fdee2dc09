"""GPU: flashmask_cache_weights against the definition in 64 bits.  Wherever nothing is cached the pages hold NaN and infinities."""
import numpy as np
import pytest
import torch

from keys_util import check_weights, ints, paged, queries, values_of
from oracle import cache_oracle, keys_oracle as orc
from serving_util import f64, raw

pytestmark = pytest.mark.gpu


def _problem(seed, lens, H, Hk, T, d, page, type, cache, packed=False, columns=None, mask="none", holes=(), hide=True):
    p = paged(seed, lens, Hk, page, d, cache, packed, columns, holes)
    rng = np.random.default_rng(seed)
    lens, N, B = np.array(lens), p["table"].shape[1] * page, len(lens)
    p["window"], bounds = 37 if mask == "window" else 0, None
    if mask == "bounds":
        n = max(N - page // 2, 1)       # keys behind the vectors' end have no interval
        lts = np.full((B, n), N)
        for b, L in enumerate(lens):
            lts[b, L // 3:L // 2], lts[b, L // 2:L * 3 // 4] = L // 2, L * 3 // 4
        lte, uts, ute = np.full_like(lts, N), np.zeros_like(lts), np.zeros_like(lts)
        uts[:, ::3], ute[:, ::3] = lens[:, None] - T, lens[:, None] - T + (T + 1) // 2
        bounds = (lts, lte, uts, ute)
    elif mask == "random":
        bounds = rng.integers(-2, N + 3, (4, B, N))
    p["bounds"], p["q"] = bounds, queries(seed, B, H, T, d, type, packed)
    if hide:            # keys that no row sees are no numbers either
        table = p["table"].cpu().numpy()
        for b, L in enumerate(lens):
            for j in range(min(L, N)):
                at = cache_oracle.place(table, len(p["k_cache"]), page, b, j)
                if at is not None and not any(cache_oracle.visible(L, t, T, j, p["window"], None if bounds is None else [x[b] for x in bounds])
                                              for t in range(T)):
                    p["k_cache"][at[0], :, at[1]] = torch.nan
    return p


def _run(p, decay, places=None, before=True, in_place=False):
    import paper_2410_01359_amd as fm
    B, H, T, d = p["q"].shape
    Hk = p["k_cache"].shape[1]
    places = places or p["table"].shape[1] * p["k_cache"].shape[2]
    bounds = None if p["bounds"] is None else [np.asarray(x) for x in p["bounds"]]
    k, _ = values_of(p)
    table, lens = p["table"].cpu().numpy(), p["lens"].cpu().numpy()
    visible_k = np.where(np.isfinite(k), k, 0)
    lse = cache_oracle.decode(f64(p["q"]), visible_k, visible_k, table, lens, d ** -0.5, p["window"], bounds)[1].astype(np.float32)
    gen = torch.Generator(device="cuda").manual_seed(5)
    old = torch.rand((B, Hk, places), device="cuda", generator=gen)
    start = old.clone() if in_place else torch.full_like(old, -3.0)
    out = old if in_place else start.clone()
    want = orc.cache_weights(f64(p["q"]), visible_k, table, lens, lse, d ** -0.5, f64(old) if before else None, decay, f64(start), p["window"], bounds)
    got = fm.flashmask_cache_weights(p["q"], p["k_cache"], p["v_cache"], p["table"], p["lens"], torch.tensor(lse, device="cuda"), d ** -0.5,
                                     old if before else None, out=None if in_place else out, decay=decay,
                                     bounds=None if bounds is None else tuple(ints(x) for x in bounds), window=p["window"], k_scale=p["k_scale"],
                                     v_scale=p["v_scale"])
    assert got is out
    # the old weight's product and sum are a rounding each
    check_weights(got, want[0], want[1], want[2] + 2, d)
    for b, n in enumerate(lens):
        assert torch.equal(got[b, :, max(int(n), 0):], start[b, :, max(int(n), 0):]), "places behind a sequence changed"
    return got


CASES = [
    # lens, H, Hk, T, d, page, columns
    ([1], 1, 1, 1, 64, 16, None),
    ([0, 1, 2, 15, 16, 17, 31, 33], 4, 4, 1, 128, 16, None),
    ([5, 0, 130, 64, 333], 8, 8, 1, 128, 64, None),
    ([333, 7], 5, 1, 1, 64, 48, None),
    ([3, 100, 1, 0, 257], 8, 2, 4, 64, 32, None),           # sequences shorter than the new tokens
    ([129, 64], 40, 5, 2, 128, 16, None),                   # 16 query rows to a K/V head
    ([300, 9], 18, 2, 2, 128, 256, None),                   # 18
    ([70, 200], 32, 2, 5, 64, 16, None),                    # 80
    ([1025, 40, 0, 2111, 1], 8, 2, 1, 128, 64, None),       # several chunks
    ([1100, 64], 2, 1, 33, 64, 16, 90),                     # rows of the table beyond what is used
]


@pytest.mark.parametrize("type,cache", [("bf16", "bf16"), ("f16", "f16"), ("bf16", "e4m3"), ("f16", "e4m3")])
@pytest.mark.parametrize("case", range(len(CASES)))
def test_against_the_definition(case, type, cache):
    lens, H, Hk, T, d, page, columns = CASES[case]
    _run(_problem(case, lens, H, Hk, T, d, page, type, cache, packed=case % 2 == 1, columns=columns), (1.0, 0.75, 0.0)[case % 3])


@pytest.mark.parametrize("type,cache", [("bf16", "bf16"), ("f16", "e4m3")])
@pytest.mark.parametrize("mask", ["window", "bounds", "random"])
@pytest.mark.parametrize("case", [1, 2, 4, 5, 6, 7, 9])
def test_masks(case, mask, type, cache):
    lens, H, Hk, T, d, page, columns = CASES[case]
    _run(_problem(100 + case, lens, H, Hk, T, d, page, type, cache, packed=case % 2 == 0, columns=columns, mask=mask), 0.5)


@pytest.mark.parametrize("places", [1, 50, 64, 100, 400])
def test_more_or_fewer_places_than_the_table(places):
    _run(_problem(3, [333, 7, 60], 4, 2, 3, 64, 16, "bf16", "bf16"), 0.9, places)


def test_pages_that_are_missing():
    _run(_problem(4, [100, 40, 64], 4, 2, 2, 64, 16, "bf16", "bf16", holes=((0, 1, -1), (0, 6, 10 ** 6), (1, 2, -7), (2, 0, -1))), 0.5)


def test_lengths_beyond_the_table_and_below_zero():
    p = _problem(5, [64, 30], 2, 2, 2, 64, 16, "bf16", "bf16", hide=False)
    p["lens"] = ints([90, -4])      # rows 88 and 89 see all that the table has
    _run(p, 0.5)


@pytest.mark.parametrize("decay,before", [(1.0, True), (0.0, True), (0.5, False)])
def test_weights_that_are_not_read(decay, before):
    """NaN in old weights that a call has no use for stays out: of the new tokens' places, and all of them without a decay."""
    import paper_2410_01359_amd as fm
    p = paged(6, [40, 100], 2, 16, 64, "bf16")
    q, lse = queries(6, 2, 4, 3, 64, "bf16"), torch.full((2, 4, 3), 4.0, device="cuda")
    old = torch.ones((2, 2, 112), device="cuda")
    for b, n in enumerate((40, 100)):
        old[b, :, n - 3:] = torch.nan
    if decay == 0:
        old[:] = torch.nan
    got = fm.flashmask_cache_weights(q, p["k_cache"], p["v_cache"], p["table"], p["lens"], lse, 0.125, old if before else None, decay=decay,
                                     out=torch.zeros_like(old))
    assert torch.isfinite(got).all()


def test_in_place_and_the_same_bits():
    p = _problem(8, [1300, 77], 16, 4, 2, 128, 32, "bf16", "bf16")
    a, b = _run(p, 0.5, in_place=True), _run(p, 0.5)
    assert torch.equal(a[0, :, :1300], b[0, :, :1300]) and torch.equal(a[1, :, :77], b[1, :, :77])


def test_a_new_tensor_is_zero_behind_the_sequences():
    import paper_2410_01359_amd as fm
    p = paged(9, [20, 0], 1, 16, 64, "f16")
    got = fm.flashmask_cache_weights(queries(9, 2, 2, 1, 64, "f16"), p["k_cache"], p["v_cache"], p["table"], p["lens"],
                                     torch.zeros((2, 2, 1), device="cuda"), 0.125)
    assert got.shape == (2, 1, 32) and (got[0, 0, 20:] == 0).all() and (got[1] == 0).all() and (got[0, 0, :20] > 0).all()


def test_every_row_gives_one():
    """With lse of flashmask_decode: what all keys of a sequence get together is the number of its rows."""
    import paper_2410_01359_amd as fm
    lens, H, Hk, T, d = [5000, 333, 64, 1], 8, 2, 3, 128
    p = paged(10, lens, Hk, 64, d, "bf16")
    q = queries(10, 4, H, T, d, "bf16")
    _, lse = fm.flashmask_decode(q, p["k_cache"], p["v_cache"], p["table"], p["lens"], d ** -0.5)
    got = fm.flashmask_cache_weights(q, p["k_cache"], p["v_cache"], p["table"], p["lens"], lse, d ** -0.5)
    rows = np.array([H // Hk * min(T, n) for n in lens])
    # lse's and the exponents' errors, of 32 bits
    assert np.abs(f64(got.double().sum(-1)) - rows[:, None]).max() <= rows.max() * 4e-5


def test_on_a_stream_of_its_own_and_in_a_graph():
    import paper_2410_01359_amd as fm
    p = _problem(11, [600, 1200], 8, 2, 2, 64, 16, "bf16", "bf16", hide=False)
    lse = torch.full((2, 8, 2), 5.0, device="cuda")
    before, out = torch.rand((2, 2, 1200), device="cuda"), torch.zeros((2, 2, 1200), device="cuda")

    def call():
        return fm.flashmask_cache_weights(p["q"], p["k_cache"], p["v_cache"], p["table"], p["lens"], lse, 0.125, before, out=out, decay=0.5)

    want = call().clone()
    torch.cuda.synchronize()
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        call()
    for n in (1, 2, 3):
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want), n
    assert raw(p["k_cache"]).shape[0] > 0


@pytest.mark.parametrize("B,long", [(64, 900), (65, 1300), (130, 1100), (512, 300), (520, 700)])
@pytest.mark.parametrize("mask", ["none", "window"])
def test_more_sequences_than_lanes(B, long, mask):
    """Lengths are added up 64 sequences at a time, up to 512; of more, every sequence has its own chunks."""
    rng = np.random.default_rng(B)
    lens = rng.integers(0, 40, B)
    lens[0], lens[B // 2], lens[-1] = long, 64, long // 2
    _run(_problem(B, lens, 2, 1, 1, 64, 16, "bf16", "bf16", mask=mask, hide=False), 0.5)


def test_many_long_sequences():
    """More chunks than one to a sequence beyond 512 sequences: 10000 keys are two of 8192."""
    lens = np.full(513, 3)
    lens[7] = 10000
    _run(_problem(20, lens, 1, 1, 1, 64, 2048, "bf16", "bf16", hide=False), 0.5)


@pytest.mark.parametrize("type,cache", [("bf16", "bf16"), ("f16", "e4m3")])
def test_more_rows_than_lie_in_lds(type, cache):
    """300 and 2048 query rows to a K/V head."""
    _run(_problem(21, [400, 33], 12, 1, 25, 128, 64, type, cache, mask="bounds"), 0.5)
    _run(_problem(22, [300], 8, 1, 256, 64, 16, type, cache, hide=False), 0.5)


MANY_ROWS = [
    # lens, H, Hk, T, d, page: more query rows than a workgroup holds at a time, more new tokens than a word has bits, few keys to share
    ([150, 64, 3, 0], 3, 1, 100, 64, 16),
    ([300, 65], 8, 1, 64, 64, 48),
    ([520, 40], 4, 2, 256, 64, 64),
    ([90, 61, 1], 16, 2, 63, 128, 32),
    ([40, 200], 34, 2, 1, 128, 16),
]


@pytest.mark.parametrize("type,cache", [("bf16", "bf16"), ("f16", "e4m3")])
@pytest.mark.parametrize("mask", ["none", "window", "bounds", "random"])
@pytest.mark.parametrize("case", range(len(MANY_ROWS)))
def test_many_rows(case, mask, type, cache):
    lens, H, Hk, T, d, page = MANY_ROWS[case]
    _run(_problem(200 + case, lens, H, Hk, T, d, page, type, cache, packed=case % 2 == 0, mask=mask), 0.5, in_place=case == 1)


def test_a_window_at_the_seam_of_two_panels():
    """More sequences than are dealt out in pieces of one size: each is one piece, whose live steps are few on both sides of key 4096.  They all
    have the pages of the first, and its weights."""
    import paper_2410_01359_amd as fm
    B, T = 520, 20
    one = _problem(30, [4166], 1, 1, T, 64, 16, "bf16", "bf16", hide=False)
    one["window"] = 100
    want = _run(one, 0.5, before=False)
    gen = torch.Generator(device="cuda").manual_seed(1)
    k, _ = values_of(one)
    k = np.where(np.isfinite(k), k, 0)
    lse = cache_oracle.decode(f64(one["q"]), k, k, one["table"].cpu().numpy(), [4166], 0.125, 100, None)[1].astype(np.float32)
    more = [x.expand(B, *x.shape[1:]).contiguous() for x in (one["q"], one["table"], torch.tensor(lse, device="cuda"))]
    old = torch.rand((B, 1, 4176), device="cuda", generator=gen)
    got = fm.flashmask_cache_weights(more[0], one["k_cache"], one["v_cache"], more[1], one["lens"].expand(B).contiguous(), more[2], 0.125, old.clone(),
                                     decay=1.0, window=100)
    assert (got[:, :, :4000] == old[:, :, :4000]).all()
    new = torch.where(torch.arange(4176, device="cuda") < 4166 - T, old, 0)[:, :, :4166]
    # Both are sums of the same 20 numbers in orders of their own: 19 additions each, off by half a step (2^-24) of what they give, which is no more than
    # the sum; the old weight's addition is one more, of both together.
    size, error = want[:, :, :4166].double(), got[:, :, :4166].double() - new.double() - want[:, :, :4166].double()
    assert (error.abs() <= 2.0 ** -24 * 1.001 * (39 * size + new)).all()
