"""GPU: flashmask_cache_evict against the plain definition: every output exactly."""
import numpy as np
import pytest
import torch

from keys_util import ints, paged, spare_pages
from oracle import keys_oracle as orc
from serving_util import f64, raw

pytestmark = pytest.mark.gpu


def _weights(kind, B, heads, columns, seed):
    rng = np.random.default_rng(seed)
    w = np.exp(2 * rng.standard_normal((B, heads, columns))).astype(np.float32)
    if kind == "few":               # a few values many times over, zeros of both signs among them
        w = rng.choice(np.array([0.0, -0.0, 1.0, 1.0 + 2.0 ** -23, 3.0], np.float32), w.shape)
    elif kind == "odd":             # anything that a 32-bit number can be
        w = rng.integers(0, 1 << 32, w.shape, dtype=np.uint64).astype(np.uint32).view(np.float32)
        w[:, :, ::7], w[:, :, 1::9], w[:, :, 2::11] = np.nan, np.inf, -np.inf
    elif kind == "same":
        w[:] = 0.25
    return w


def _check(p, weights, new_table, keep, first, recent, **more):
    import paper_2410_01359_amd as fm
    old = [f64(p[n]) for n in ("k_cache", "v_cache")]
    kept_raw = [raw(p[n]).clone() for n in ("k_cache", "v_cache")]
    table, lens = p["table"].cpu().numpy(), p["lens"].cpu().numpy()
    want = orc.evict(old, table, lens, weights, new_table, keep, first, recent)
    got = fm.flashmask_cache_evict(p["k_cache"], p["v_cache"], p["table"], p["lens"], torch.tensor(weights, device="cuda"), ints(new_table), keep,
                                   first=first, recent=recent, k_scale=p["k_scale"], v_scale=p["v_scale"], **more)
    assert np.array_equal(got[3].cpu().numpy(), want[4]), "kept"
    assert np.array_equal(got[0].cpu().numpy(), want[1]) and np.array_equal(got[1].cpu().numpy(), want[2])
    assert np.array_equal(got[2].cpu().numpy(), want[3], equal_nan=True), "weights"
    for n, before, after in zip(("k_cache", "v_cache"), kept_raw, want[0]):
        assert np.array_equal(f64(p[n]), after, equal_nan=True), n
        fresh = np.unique(new_table[(new_table >= 0) & (new_table < len(before))])
        stays = np.setdiff1d(np.arange(len(before)), fresh)
        assert torch.equal(raw(p[n])[stays], before[stays]), "a page that was not given changed"
    return got


def _new_table(p, keep, columns=None):
    B, page = p["table"].shape[0], p["k_cache"].shape[2]
    need = -(-keep // page)
    pages = spare_pages(p)[:B * need].reshape(B, need)
    return np.concatenate((pages, np.full((B, (columns or need) - need), -1)), 1)


CASES = [
    # lens, heads, page, d, keep, first, recent
    ([2], 1, 16, 64, 1, 0, 0),
    ([40, 16, 0, 17, 16], 2, 16, 128, 16, 0, 0),
    ([100, 33, 64, 65, 1], 3, 16, 64, 33, 4, 9),
    ([333, 200], 8, 64, 128, 150, 0, 150),          # nothing but the last ones
    ([333, 64], 1, 32, 64, 40, 40, 0),              # nothing but the first ones
    ([129, 700], 4, 48, 128, 128, 1, 1),
    ([1500, 1024, 1025], 2, 128, 64, 1024, 4, 100),
    ([5000, 30, 2100], 2, 256, 64, 999, 0, 64),
]


@pytest.mark.parametrize("cache", ["bf16", "f16", "e4m3"])
@pytest.mark.parametrize("shared", [False, True])
@pytest.mark.parametrize("case", range(len(CASES)))
def test_against_the_definition(case, shared, cache):
    lens, heads, page, d, keep, first, recent = CASES[case]
    B = len(lens)
    p = paged(case, lens, heads, page, d, cache, packed=case % 2 == 1, spare=B * (-(-keep // page)) + 2)
    weights = _weights("plain", B, 1 if shared else heads, p["table"].shape[1] * page, case)
    _check(p, weights, _new_table(p, keep, None if case % 2 else -(-keep // page) + 3), keep, first, recent)


@pytest.mark.parametrize("kind", ["few", "odd", "same"])
@pytest.mark.parametrize("case", [1, 2, 5, 6, 7])
def test_equal_and_odd_weights(case, kind):
    lens, heads, page, d, keep, first, recent = CASES[case]
    B = len(lens)
    p = paged(20 + case, lens, heads, page, d, "bf16", spare=B * (-(-keep // page)))
    _check(p, _weights(kind, B, heads, p["table"].shape[1] * page, case), _new_table(p, keep), keep, first, recent)


@pytest.mark.parametrize("kind", ["plain", "few", "odd", "same"])
@pytest.mark.parametrize("lens,heads,keep,first,recent", [([40000, 100, 17001], 2, 9000, 4, 500), ([16500, 16640], 1, 16400, 0, 0), ([30000], 1, 700, 300, 400),
                                                          ([140000], 1, 20000, 1, 1), ([20000, 5], 1, 1, 0, 0)])
def test_long_rows(lens, heads, keep, first, recent, kind):
    """Rows that several workgroups share."""
    B = len(lens)
    p = paged(40, lens, heads, 256, 64, "e4m3", spare=B * -(-keep // 256))
    p["k_scale"], p["v_scale"] = (torch.ones(heads, device="cuda") for _ in range(2))
    _check(p, _weights(kind, B, heads, p["table"].shape[1] * 256, len(lens)), _new_table(p, keep), keep, first, recent)


def test_a_long_row_with_fewer_weights_than_places():
    p = paged(41, [40000], 1, 256, 64, "e4m3", spare=80)
    weights = _weights("plain", 1, 1, 17000, 6)
    weights[0, 0, ::3] *= -1
    _check(p, weights, _new_table(p, 20000), 20000, 0, 10)


@pytest.mark.parametrize("heads,B", [(129, 1), (1, 130)])
def test_many_long_rows(heads, B):
    """More than are shared."""
    lens = [16500] + [20] * (B - 1)
    p = paged(42, lens, heads, 4096, 64, "e4m3", spare=2 * B)
    _check(p, _weights("plain", B, heads, 20480, 7), _new_table(p, 5000), 5000, 3, 30)


@pytest.mark.parametrize("columns", [1, 30, 64, 90, 500])
def test_more_or_fewer_weights_than_places(columns):
    """Places without a weight have 0, and a negative weight is lighter."""
    p = paged(30, [100, 20, 96], 2, 16, 64, "bf16", spare=9)
    weights = _weights("plain", 3, 2, columns, 1)
    weights[:, :, ::5] *= -1
    _check(p, weights, _new_table(p, 40), 40, 2, 3)


def test_pages_that_are_missing():
    """Kept tokens without a page become zeros, places without a page are not written."""
    p = paged(31, [100, 64, 50], 2, 16, 64, "bf16", spare=9, holes=((0, 2, -1), (0, 5, 1 << 20), (1, 0, -3)))
    fresh = _new_table(p, 40)
    fresh[1, 1], fresh[0, 2] = -1, 1 << 30
    _check(p, _weights("plain", 3, 2, 112, 2), fresh, 40, 17, 9)


def test_lengths_beyond_the_table_and_below_zero():
    p = paged(32, [64, 64, 64], 1, 16, 64, "bf16", spare=6)
    p["lens"] = ints([90, -5, 70])
    _check(p, _weights("plain", 3, 1, 64, 3), _new_table(p, 32), 32, 0, 4)


def test_twice():
    """What was evicted goes on: again, from its new pages and weights."""
    p = paged(33, [200, 90], 2, 16, 64, "f16", spare=2 * 6 + 2 * 3)
    pages = spare_pages(p)
    got = _check(p, _weights("plain", 2, 2, 208, 4), pages[:12].reshape(2, 6), 90, 4, 20)
    again = {**p, "table": got[0], "lens": got[1]}
    _check(again, got[2].cpu().numpy(), pages[12:].reshape(2, 3), 48, 4, 20)


@pytest.mark.parametrize("long", [3000, 17000])
def test_on_a_stream_of_its_own_and_in_a_graph(long):
    import paper_2410_01359_amd as fm
    p = paged(34, [long, 500, 20], 2, 32, 64, "bf16", spare=3 * 8)
    places = p["table"].shape[1] * 32
    weights, fresh = torch.tensor(_weights("plain", 3, 2, places, 5), device="cuda"), ints(_new_table(p, 256))
    ws = torch.empty(fm.flashmask_cache_evict_workspace_bytes(3, 2, places), dtype=torch.uint8, device="cuda")

    def call():
        return fm.flashmask_cache_evict(p["k_cache"], p["v_cache"], p["table"], p["lens"], weights, fresh, 256, first=4, recent=64, workspace=ws)

    want = [x.clone() for x in call()] + [raw(p["k_cache"]).clone(), raw(p["v_cache"]).clone()]
    torch.cuda.synchronize()
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        got = call()
    for _ in range(3):
        for x in got:
            x.fill_(-7)
        raw(p["k_cache"])[fresh[:2].long().flatten()] = 0       # the third sequence is not evicted from: its pages are not written
        ws.fill_(255)
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip([*got, raw(p["k_cache"]), raw(p["v_cache"])], want):
            assert torch.equal(a, b)
