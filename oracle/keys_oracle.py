"""Plain fp64 definitions of the operators that weigh a cache's keys, drop the light ones, and verify trees of drafted tokens.

TEST INFRASTRUCTURE, as cache_oracle.py is: NumPy in 64 bits, sequence by sequence, sharing no code with the GPU path.
"""
from __future__ import annotations

import numpy as np

from .cache_oracle import place, visible


def hidden(bounds, i, j):
    """Whether bounds (lts, lte, uts, ute) hide key j from row i; keys behind the vectors' end have no interval."""
    if bounds is None or j >= len(bounds[0]):
        return False
    lts, lte, uts, ute = (int(x[j]) for x in bounds)
    return lts <= i < lte or uts <= i < ute


def weights(q, k, lse, bounds, scale, first_row=0):
    """[B,Hk,N]: the weight that each key gets from the rows that see it, and for tolerances the same of the terms times
    their size |lse| + scale * sum |q||k|, and the number of terms."""
    q, k, lse = (np.asarray(x, np.float64) for x in (q, k, lse))
    B, H, N, _ = q.shape
    Hk = k.shape[1]
    out, size, terms = (np.zeros((B, Hk, N)) for _ in range(3))
    i, j = np.arange(N)[:, None], np.arange(N)
    for b in range(B):
        lts, lte, uts, ute = (np.asarray(x[b], np.int64) for x in bounds)
        seen = ~(((lts <= i) & (i < lte)) | ((uts <= i) & (i < ute))) & (i >= first_row)
        for h in range(H):
            hk = h // (H // Hk)
            live = seen & ~np.isneginf(lse[b, h])[:, None]
            logit = np.where(live, (q[b, h] @ k[b, hk].T) * scale - lse[b, h][:, None], -np.inf)
            p = np.exp(logit)
            out[b, hk] += p.sum(0)
            grown = np.abs(q[b, h]) @ np.abs(k[b, hk]).T * scale + np.abs(np.where(np.isfinite(lse[b, h]), lse[b, h], 0))[:, None]
            size[b, hk] += (p * grown).sum(0)
            terms[b, hk] += live.sum(0)
    return out, size, terms


def cache_weights(q, k_cache, table, lens, lse, scale, before, decay, weights, window=0, bounds=None):
    """weights [B,Hk,n] after the new tokens' call, and size and terms as above."""
    q, k_cache, lse = (np.asarray(x, np.float64) for x in (q, k_cache, lse))
    B, H, T, _ = q.shape
    pages, Hk, page, _ = k_cache.shape
    out = np.array(weights, np.float64)
    size, terms = np.zeros(out.shape), np.zeros(out.shape)
    for b in range(B):
        length = max(int(lens[b]), 0)
        mine = None if bounds is None else [x[b] for x in bounds]
        for j in range(min(length, table.shape[1] * page, out.shape[2])):
            old = decay * np.asarray(before[b, :, j], np.float64) if before is not None and decay > 0 and j < length - T else 0.0
            out[b, :, j] = old
            at = place(table, pages, page, b, j)
            if at is None:
                continue
            for t in range(T):
                if not visible(length, t, T, j, window, mine):
                    continue
                for h in range(H):
                    hk = h // (H // Hk)
                    if np.isneginf(lse[b, h, t]):
                        continue
                    key = k_cache[at[0], hk, at[1]]
                    p = np.exp(q[b, h, t] @ key * scale - lse[b, h, t])
                    out[b, hk, j] += p
                    size[b, hk, j] += p * (np.abs(q[b, h, t]) @ np.abs(key) * scale + abs(lse[b, h, t]))
                    terms[b, hk, j] += 1
    return out, size, terms


def ancestors(parents):
    """Each token's line: its ancestors from the first, and itself."""
    lines = []
    for t, p in enumerate(parents):
        lines.append((lines[p] if 0 <= p < t else []) + [t])
    return lines


def tree_visible(length, T, lines, t, j, window=0, bounds=None):
    """Whether drafted token t sees the key in place j."""
    start = length - T
    i = start + len(lines[t]) - 1
    if start + t < 0 or j >= length:
        return False
    u = j - start
    if u >= 0:
        if u not in lines[t]:
            return False
        at = start + len(lines[u]) - 1
    else:
        at = j
    return not (window > 0 and at <= i - window) and not hidden(bounds, i, j)


def decode_tree(q, k_cache, v_cache, table, lens, parents, scale, window=0, bounds=None):
    """As cache_oracle.decode: out, lse, sum of p |v|, largest scale * sum |q||k|."""
    q, k_cache, v_cache = (np.asarray(x, np.float64) for x in (q, k_cache, v_cache))
    B, H, T, d = q.shape
    pages, heads, page, _ = k_cache.shape
    out, mass = np.zeros((B, H, T, d)), np.zeros((B, H, T, d))
    lse, size = np.full((B, H, T), -np.inf), np.zeros((B, H, T))
    for b in range(B):
        length, lines = max(int(lens[b]), 0), ancestors(parents[b])
        mine = None if bounds is None else [x[b] for x in bounds]
        places = [(j, place(table, pages, page, b, j)) for j in range(min(length, table.shape[1] * page))]
        for t in range(T):
            at = [x for j, x in places if x is not None and tree_visible(length, T, lines, t, j, window, mine)]
            if not at:
                continue
            number, slot = (np.array(x) for x in zip(*at))
            for h in range(H):
                k, v = (c[number, h // (H // heads), slot] for c in (k_cache, v_cache))
                s = k @ q[b, h, t] * scale
                top = s.max()
                p = np.exp(s - top)
                total = p.sum()
                out[b, h, t], mass[b, h, t] = p @ v / total, p @ np.abs(v) / total
                lse[b, h, t] = top + np.log(total)
                size[b, h, t] = (np.abs(k) @ np.abs(q[b, h, t])).max() * scale
    return out, lse, mass, size


def accepted(path, T):
    """The part of a path that counts."""
    line = []
    for t in path:
        if not 0 <= t < T or (line and t <= line[-1]):
            break
        line.append(int(t))
    return line


def accept(pools, table, lens, T, paths):
    """(pools, lens) after the accepted tokens moved."""
    pools = [np.array(p) for p in pools]
    num_pages, _, page, _ = pools[0].shape
    new = np.array(lens)
    for b, length in enumerate(lens):
        start = int(length) - T
        if start < 0:
            continue
        line = accepted(paths[b], T)
        new[b] = start + len(line)
        for p in pools:
            rows = [place(table, num_pages, page, b, start + t) for t in line]
            rows = [0 if x is None else p[x[0], :, x[1]].copy() for x in rows]
            for i, (t, row) in enumerate(zip(line, rows)):
                to = place(table, num_pages, page, b, start + i)
                if t != i and to is not None:
                    p[to[0], :, to[1]] = row
    return pools, new


def select(weights, keep, first, recent):
    """Places of a row of weights that stay, in order."""
    n = len(weights)
    if n <= keep:
        return list(range(n))
    middle = range(first, n - recent)
    # NaN is lighter than everything else
    heavy = sorted(middle, key=lambda j: (np.isnan(weights[j]), 0 if np.isnan(weights[j]) else -weights[j], j))[:keep - first - recent]
    return list(range(first)) + sorted(heavy) + list(range(n - recent, n))


def evict(pools, table, lens, weights, new_table, keep, first, recent):
    """(pools, table, lens, weights, kept) afterwards; pools: keys, values."""
    pools = [np.array(p) for p in pools]
    num_pages, Hk, page, _ = pools[0].shape
    B, heads, columns = weights.shape
    rows, new_lens = np.array(table), np.array(lens)
    out, kept = np.zeros(weights.shape, weights.dtype), np.full((B, heads, keep), -1, np.int32)
    for b in range(B):
        n = min(max(int(lens[b]), 0), table.shape[1] * page)
        for h in range(heads):
            row = np.zeros(n, weights.dtype)
            row[:min(n, columns)] = weights[b, h, :min(n, columns)]
            at = select(row, keep, first, recent)
            kept[b, h, :len(at)] = at
            out[b, h, :min(len(at), columns)] = row[at][:columns]
        if n <= keep:
            continue
        used = -(-keep // page)
        rows[b], rows[b, :used], new_lens[b] = -1, new_table[b, :used], keep
        for p in pools:
            old = p.copy()
            for h in range(Hk):
                for i, j in enumerate(kept[b, h if heads > 1 else 0]):
                    source, to = place(table, num_pages, page, b, int(j)), place(new_table, num_pages, page, b, i)
                    if to is not None:
                        p[to[0], h, to[1]] = 0 if source is None else old[source[0], h, source[1]]
    return pools, rows, new_lens, out, kept
