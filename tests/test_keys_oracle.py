"""No GPU: the definitions of the weights of keys, of eviction and of trees of drafted tokens against what must hold of them."""
import numpy as np
import pytest

from oracle import cache_oracle, flashmask_oracle, keys_oracle as orc


def _paged(rng, lens, heads, page, d, columns):
    """Caches, table."""
    B = len(lens)
    order = rng.permutation(B * columns + 2)
    table = order[:B * columns].reshape(B, columns)
    return rng.standard_normal((2, B * columns + 2, heads, page, d)), table


def test_weights_are_the_columns_of_the_attention_matrix():
    rng = np.random.default_rng(0)
    N, d = 23, 8
    q, k, v = rng.standard_normal((3, 1, 1, N, d))
    lts, lte, uts, ute = rng.integers(0, N, (4, 1, N))
    lse = flashmask_oracle.forward(q[0, 0], k[0, 0], v[0, 0], lts[0], lte[0], uts[0], ute[0], 0.3)[1][None, None]
    seen = np.array([[not (lts[0, j] <= i < lte[0, j] or uts[0, j] <= i < ute[0, j]) for j in range(N)] for i in range(N)])
    want = np.zeros(N)
    for i in range(N):
        if seen[i].any():
            e = np.where(seen[i], np.exp(k[0, 0] @ q[0, 0, i] * 0.3), 0)
            want += e / e.sum()
    got, _, terms = orc.weights(q, k, lse, (lts, lte, uts, ute), 0.3)
    assert np.allclose(got[0, 0], want, atol=1e-12) and (terms[0, 0] == seen.sum(0)).all()
    # every row that sees something gives 1 in all
    assert np.isclose(got.sum(), seen.any(1).sum())


def test_weights_of_grouped_heads_and_last_rows():
    rng = np.random.default_rng(1)
    N = 12
    q, k = rng.standard_normal((1, 4, N, 8)), rng.standard_normal((1, 2, N, 8))
    none = tuple(np.zeros((1, N), int) for _ in range(4))
    lse = rng.standard_normal((1, 4, N))
    all_rows, last = orc.weights(q, k, lse, none, 0.5)[0], orc.weights(q, k, lse, none, 0.5, first_row=9)[0]
    head = [orc.weights(q[:, h:h + 1], k[:, h // 2:h // 2 + 1], lse[:, h:h + 1], none, 0.5)[0][0, 0] for h in range(4)]
    assert np.allclose(all_rows[0], [head[0] + head[1], head[2] + head[3]])
    assert (last < all_rows).all() and np.allclose(last[0, 0], sum(np.exp(k[0, 0] @ q[0, h, i] * 0.5 - lse[0, h, i]) for h in (0, 1) for i in (9, 10, 11)))


def test_cache_weights_are_those_of_the_sequence():
    rng = np.random.default_rng(2)
    lens, page, T = [37, 5], 16, 3
    (k, v), table = _paged(rng, lens, 2, page, 8, 3)
    q = rng.standard_normal((2, 4, T, 8))
    lse = cache_oracle.decode(q, k, v, table, lens, 0.4, window=9)[1]
    before = rng.random((2, 2, 48))
    start = np.full((2, 2, 48), 7.0)
    got, _, terms = orc.cache_weights(q, k, table, lens, lse, 0.4, before, 0.5, start, window=9)
    for b, n in enumerate(lens):
        assert (got[b, :, n:] == 7).all()
        old = np.where(np.arange(n) < n - T, 0.5 * before[b, :, :n], 0)
        assert np.allclose((got[b, :, :n] - old).sum(-1), 2 * T)      # two heads, T rows
        assert terms[b, 0, 0] == (0 if n > 9 + T else 2 * T)


@pytest.mark.parametrize("window", [0, 4])
def test_a_tree_of_one_line_is_a_sequence(window):
    rng = np.random.default_rng(3)
    lens, T = [20, 6, 3], 5
    (k, v), table = _paged(rng, lens, 1, 16, 8, 2)
    q = rng.standard_normal((3, 2, T, 8))
    chain = np.tile(np.arange(T) - 1, (3, 1))
    for got, want in zip(orc.decode_tree(q, k, v, table, lens, chain, 0.4, window), cache_oracle.decode(q, k, v, table, lens, 0.4, window)):
        assert np.allclose(got, want)


def test_a_path_of_a_tree_is_a_sequence_of_its_own():
    """A token of a tree has the result that it has where its line alone was drafted."""
    rng = np.random.default_rng(4)
    n, parents = 21, np.array([-1, 0, 0, 7, 1, 2, -1, 4])      # 7 is not ahead of token 3
    T = len(parents)
    (k, v), table = _paged(rng, [n], 1, 16, 8, 2)
    bounds = tuple(x[None] for x in (np.full(n, n), np.full(n, n), np.zeros(n, int), np.zeros(n, int)))
    bounds[0][0, 3], bounds[0][0, 15] = 14, 15                  # key 3 hidden from row 14 on
    q = rng.standard_normal((1, 1, T, 8))
    out, lse, _, _ = orc.decode_tree(q, k, v, table, [n], parents[None], 0.4, 6, bounds)
    lines = orc.ancestors(parents)
    assert lines[5] == [0, 2, 5] and lines[3] == [3] and lines[7] == [0, 1, 4, 7]
    start = n - T
    for t, line in enumerate(lines):
        place = [cache_oracle.place(table, len(k), 16, 0, j) for j in list(range(start)) + [start + u for u in line]]
        keys, values = (np.zeros((3, 1, 16, 8)) for _ in range(2))
        for j, (p, slot) in enumerate(place):
            keys[j // 16, 0, j % 16], values[j // 16, 0, j % 16] = k[p, 0, slot], v[p, 0, slot]
        mine = tuple(np.concatenate((x[0, :start], x[0, [start + u for u in line]]))[None] for x in bounds)
        want = cache_oracle.decode(q[:, :, t:t + 1], keys, values, np.arange(3)[None], [len(place)], 0.4, 6, mine)
        assert np.allclose(out[0, 0, t], want[0][0, 0, 0]) and np.isclose(lse[0, 0, t], want[1][0, 0, 0])


def test_accepted_paths():
    assert orc.accepted([0, 3, 4, -1, 5], 6) == [0, 3, 4]
    assert orc.accepted([2, 2], 6) == [2] and orc.accepted([6], 6) == [] and orc.accepted([1, 0], 6) == [1]
    pool = np.arange(2 * 16, dtype=float).reshape(2, 1, 16, 1)
    table = np.array([[1, 0]])
    (got,), lens = orc.accept([pool], table, [20], 6, [[0, 3, 5]])
    assert lens[0] == 17
    sequence = np.concatenate((got[1, 0, :, 0], got[0, 0, :, 0]))[:17]
    assert (sequence == [*range(16, 30), 30, 1, 3]).all()       # places 14, 17 and 19 behind the first 14


def test_selection():
    w = np.array([5, 1, 3, 3, 3, np.nan, -np.inf, 2, 0, 9.0])
    assert orc.select(w, 10, 0, 0) == list(range(10))
    assert orc.select(w, 3, 0, 0) == [0, 2, 9] and orc.select(w, 4, 0, 0) == [0, 2, 3, 9]
    assert orc.select(w, 5, 2, 1) == [0, 1, 2, 3, 9] and orc.select(w, 9, 0, 0) == [0, 1, 2, 3, 4, 6, 7, 8, 9]
    assert orc.select(w, 4, 1, 3) == [0, 7, 8, 9]


def test_eviction():
    rng = np.random.default_rng(5)
    (k, v), table = _paged(rng, [40, 16], 2, 16, 4, 3)
    k, v = (np.concatenate((x, np.zeros((2, 2, 16, 4)))) for x in (k, v))
    weights = rng.random((2, 2, 48))
    fresh = np.array([[8, 9], [-1, -1]])
    (nk, nv), rows, lens, out, kept = orc.evict((k, v), table, np.array([40, 16]), weights, fresh, 20, 2, 5)
    assert lens.tolist() == [20, 16] and rows[0].tolist() == [8, 9, -1] and (rows[1] == table[1]).all()
    assert (kept[1, :, :16] == np.arange(16)).all() and (kept[1, :, 16:] == -1).all()
    for h in range(2):
        at = kept[0, h]
        assert (np.diff(at) > 0).all() and set(at) >= {0, 1, 35, 36, 37, 38, 39}
        gone, heavy = np.setdiff1d(np.arange(40), at), np.setdiff1d(at, [0, 1, 35, 36, 37, 38, 39])
        assert weights[0, h, gone].max() < weights[0, h, heavy].min()
        assert (out[0, h, :20] == weights[0, h, at]).all() and (out[0, h, 20:] == 0).all()
        for i, j in enumerate(at):
            assert (nk[[8, 9][i // 16], h, i % 16] == k[table[0, j // 16], h, j % 16]).all()
            assert (nv[[8, 9][i // 16], h, i % 16] == v[table[0, j // 16], h, j % 16]).all()
    assert (nk[:8] == k[:8]).all()
