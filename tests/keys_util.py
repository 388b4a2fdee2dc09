"""Shared by the GPU tests of weights of keys, eviction and trees of drafted tokens."""
import numpy as np
import torch

from serving_util import TYPES, cache_of, f64, raw, rows_of

STEP = 2.0 ** -23


def ints(x):
    return torch.tensor(np.asarray(x), dtype=torch.int32, device="cuda")


def paged(seed, lens, heads, page, d, cache, packed=False, columns=None, holes=(), spare=3, junk=True):
    """k_cache, v_cache, table, lens and scales; nothing but the tokens themselves is a number.  holes: (sequence, column, entry) of the table
    that name no page."""
    rng = np.random.default_rng(seed)
    gen = torch.Generator(device="cuda").manual_seed(seed)
    lens = np.array(lens)
    counts = -(-lens.clip(0) // page)
    columns = columns or max(1, counts.max())
    counts = np.minimum(counts, columns)
    num_pages = int(counts.sum()) + spare
    order, table = rng.permutation(num_pages), np.full((len(lens), columns), -1, np.int64)
    for b, n in enumerate(counts):
        table[b, :n] = order[counts[:b].sum():counts[:b].sum() + n]
    for b, c, entry in holes:
        table[b, c] = entry
    caches = []
    for _ in range(2):
        c = cache_of(gen, cache, num_pages, heads, page, d, packed, junk=junk)
        at = rows_of(c, table, lens)
        if at is not None:
            raw(c)[at[0], :, at[1]] = raw(cache_of(gen, cache, len(at[0]), heads, 16, d)[:, :, 0].contiguous())
        caches.append(c)
    scales = [torch.rand(heads, device="cuda", generator=gen) + 0.5 for _ in range(2)] if cache == "e4m3" else [None, None]
    return {"k_cache": caches[0], "v_cache": caches[1], "table": ints(table), "lens": ints(lens), "k_scale": scales[0], "v_scale": scales[1]}


def spare_pages(problem):
    """Pages that the table does not name."""
    return np.setdiff1d(np.arange(problem["k_cache"].shape[0]), problem["table"].cpu().numpy())


def queries(seed, B, H, T, d, type, packed=False):
    gen = torch.Generator(device="cuda").manual_seed(seed + 1000)
    q = torch.randn((B, T, H, d) if packed else (B, H, T, d), device="cuda", generator=gen).to(TYPES[type])
    return q.transpose(1, 2) if packed else q


def values_of(problem):
    """Caches as the values that they stand for, in 64 bits."""
    k, v = f64(problem["k_cache"]), f64(problem["v_cache"])
    if problem["k_scale"] is not None:
        k, v = (x * f64(s)[:, None, None] for x, s in ((k, problem["k_scale"]), (v, problem["v_scale"])))
    return k, v


def weight_bound(want, size, terms, d):
    """Bound on the error of sums of exp(s - lse) in 32 bits.  s is d products added in 32 bits, off by (d + 8) steps of sum |q||k|; its
    product with the scale, lse in the log2 domain and their difference are a rounding each of a number as large as both together; the
    exponential is off by 2^-21; sums by half a step for every addition."""
    relative = (d + 16) * STEP
    return 1.05 * relative * size + (2.0 ** -21 + terms * STEP / 2) * np.abs(want) + 1e-35


def check_weights(got, want, size, terms, d, what=""):
    got = f64(got)
    excess = np.abs(got - want) - weight_bound(want, size, terms, d)
    assert np.isfinite(got).all(), f"{what}: not finite"
    at = np.unravel_index(np.argmax(excess), excess.shape)
    assert excess[at] <= 0, f"{what}{list(at)}: {got[at]} for {want[at]}"
