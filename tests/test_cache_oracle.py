"""No GPU: the fp64 definitions of the cache operators against the dense-mask oracle, closed forms and differences."""
import numpy as np
import pytest

from oracle import cache_oracle as cache
from oracle import flashmask_oracle as orc


def _paged(rng, x, page, spare=2):
    """Pages and a table that hold x [heads, N, d]."""
    heads, N, d = x.shape
    n = -(-N // page)
    order = rng.permutation(n + spare)[:n]
    pages = np.full((n + spare, heads, page, d), np.nan)
    for c, p in enumerate(order):
        rows = x[:, c * page:(c + 1) * page]
        pages[p, :, :rows.shape[1]] = rows
    return pages, order.astype(np.int32)[None]


@pytest.mark.parametrize("window", [0, 5])
@pytest.mark.parametrize("T", [1, 4])
def test_decode_is_the_last_rows_of_the_dense_forward(T, window):
    rng = np.random.default_rng(3)
    N, d, H, Hk = 37, 8, 4, 2
    q, k, v = rng.normal(size=(H, N, d)), rng.normal(size=(Hk, N, d)), rng.normal(size=(Hk, N, d))
    lts = np.where(np.arange(N) < 20, 25, N)
    lte = np.full(N, N)
    if window:
        lts = np.minimum(lts, np.arange(N) + window)
    uts, ute = np.zeros(N, int), np.arange(N)       # causal
    kp, table = _paged(rng, k, 16)
    vp = np.full_like(kp, np.nan)
    for c, p in enumerate(table[0]):
        vp[p, :, :v[:, c * 16:(c + 1) * 16].shape[1]] = v[:, c * 16:(c + 1) * 16]
    bounds = (np.where(np.arange(N) < 20, 25, N)[None], lte[None], np.zeros((1, N), int), np.zeros((1, N), int))
    out, lse, _, _ = cache.decode(q[None, :, -T:], kp, vp, table, [N], 0.3, window, bounds)
    for h in range(H):
        ref, ref_lse = orc.forward(q[h], k[h // 2], v[h // 2], lts, lte, uts, ute, 0.3)
        assert np.allclose(out[0, h], ref[-T:], atol=1e-12)
        assert np.allclose(lse[0, h], ref_lse[-T:], atol=1e-12)


def test_rows_without_keys():
    q, pages = np.ones((3, 1, 2, 4)), np.ones((2, 1, 16, 4))
    table = np.array([[0], [1], [-1]], np.int32)
    out, lse, _, _ = cache.decode(q, pages, pages, table, [0, 1, 5], 1.0)
    assert np.isneginf(lse[0]).all() and np.isneginf(lse[2]).all() and np.isneginf(lse[1, 0, 0])
    assert (out[0] == 0).all() and (out[2] == 0).all() and np.allclose(out[1, 0, 1], 1)


@pytest.mark.parametrize("interleaved", [False, True])
def test_rope_keeps_lengths_depends_on_distance_and_turns_back(interleaved):
    rng = np.random.default_rng(4)
    freqs = 100.0 ** -(np.arange(4) / 4)
    x, y = rng.normal(size=(6, 10)), rng.normal(size=(6, 10))
    at = np.array([0, 1, 5, 9, 100, -3])
    a = cache.rope(x, at, freqs, interleaved)
    assert np.array_equal(a[0], x[0]) and np.array_equal(a[:, 8:], x[:, 8:])
    assert np.allclose((a ** 2).sum(-1), (x ** 2).sum(-1))
    b = cache.rope(y, at, freqs, interleaved)
    moved = [(cache.rope(x, at + s, freqs, interleaved) * cache.rope(y, at + s, freqs, interleaved)).sum(-1) for s in (0, 7)]
    assert np.allclose(moved[0], moved[1]) and np.allclose(moved[0], (a * b).sum(-1))
    assert np.allclose(cache.rope(a, at, freqs, interleaved, backward=True), x)
    # the gradient of <w, rope(x)>, by differences
    w, amp = rng.normal(size=(6, 10)), 1.3
    grad = cache.rope(w, at, freqs, interleaved, amp, backward=True)
    for r, c in ((1, 0), (2, 3), (4, 7), (5, 9)):
        step = np.zeros_like(x)
        step[r, c] = 1e-5
        up, down = (w * cache.rope(x + s * step, at, freqs, interleaved, amp) for s in (1, -1))
        want = grad[r, c] if c < 8 else w[r, c]
        assert abs((up.sum() - down.sum()) / 2e-5 - want) < 1e-8


def test_pairs_of_both_layouts():
    x = np.arange(1.0, 5.0)[None]
    quarter = np.array([np.pi / 2, np.pi])
    assert np.allclose(cache.rope(x, [1], quarter, True), [[-2, 1, -3, -4]])
    assert np.allclose(cache.rope(x, [1], quarter, False), [[-3, -2, 1, -4]])


def test_fork_and_compact():
    pool = np.arange(6.0)[:, None] * np.ones((6, 16))
    table = np.array([[4, 1], [5, -1], [9, -7]], np.int32)
    pools, rows, lens = cache.fork([pool], table, [20, 16, 3], [0, 0, 1, 7], [-1, 2, 3, 0], 16)
    assert rows.tolist() == [[4, 1], [4, 2], [5, -1], [-1, -1]] and lens.tolist() == [20, 20, 16, 0]
    assert pools[0][:, 0].tolist() == [0, 1, 1, 3, 4, 5]
    free, count = cache.free_list(table, 6)
    assert free.tolist() == [0, 2, 3, -1, -1, -1] and count == 3
    pools, rows, used = cache.compact([pool], table)
    assert used == 3 and rows.tolist() == [[0, 1], [2, -1], [9, -7]] and pools[0][:3, 0].tolist() == [4, 1, 5]
