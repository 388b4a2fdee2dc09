"""Plain fp64 definitions of the operators around the attention call: rotary positions, the paged cache, attention of new
tokens over it, forks and compaction of its pages.

TEST INFRASTRUCTURE, as flashmask_oracle.py is: NumPy in 64 bits, sequence by sequence, sharing no code with the GPU path.
Pages are arrays indexed [page, head, token, d]; page table entries outside [0, pages) stand for "no page".
"""
from __future__ import annotations

import numpy as np


def rope(x, positions, freqs, interleaved, amp=1.0, backward=False):
    """x [..., rows, d] with its rows' first 2 len(freqs) elements turned by positions [..., rows] * freqs."""
    x = np.asarray(x, np.float64)
    half = len(freqs)
    turn = amp * np.exp((-1j if backward else 1j) * (np.asarray(positions, np.float64)[..., None] * freqs))
    out = x.copy()
    a, b = (slice(0, 2 * half, 2), slice(1, 2 * half, 2)) if interleaved else (slice(0, half), slice(half, 2 * half))
    pair = (x[..., a] + 1j * x[..., b]) * turn
    out[..., a], out[..., b] = pair.real, pair.imag
    return out


def place(table, num_pages, page, seq, position):
    """(page, slot) of a token, None where it has no place."""
    if not 0 <= seq < table.shape[0] or position < 0 or position // page >= table.shape[1]:
        return None
    entry = int(table[seq, position // page])
    return (entry, position % page) if 0 <= entry < num_pages else None


def append(cache, rows, table, page, seqs, positions):
    """The cache [pages, heads, page, d] with rows [tokens, heads, d] written to it."""
    out = np.asarray(cache, np.float64).copy()
    for n, (seq, position) in enumerate(zip(seqs, positions)):
        at = place(table, out.shape[0], page, int(seq), int(position))
        if at is not None:
            out[at[0], :, at[1]] = rows[n]
    return out


def visible(length, t, T, j, window=0, bounds=None):
    """Whether query t of T of a sequence of `length` tokens sees key j; bounds: its (lts, lte, uts, ute) vectors."""
    i = length - T + t
    if j > i or (window > 0 and j <= i - window):
        return False
    if bounds is None or j >= len(bounds[0]):
        return True
    lts, lte, uts, ute = (int(x[j]) for x in bounds)
    return not (lts <= i < lte or uts <= i < ute)


def decode(q, k_cache, v_cache, table, lens, scale, window=0, bounds=None):
    """out [B,H,T,d], lse [B,H,T] and, for tolerances, sum_j p_j |v_j| [B,H,T,d] and the largest scale * sum |q||k| [B,H,T]."""
    q, k_cache, v_cache = (np.asarray(x, np.float64) for x in (q, k_cache, v_cache))
    B, H, T, d = q.shape
    pages, heads, page, _ = k_cache.shape
    out, mass = np.zeros((B, H, T, d)), np.zeros((B, H, T, d))
    lse, size = np.full((B, H, T), -np.inf), np.zeros((B, H, T))
    for b in range(B):
        length = max(int(lens[b]), 0)
        for t in range(T):
            keys = [j for j in range(min(length, table.shape[1] * page))
                    if 0 <= table[b, j // page] < pages and visible(length, t, T, j, window, None if bounds is None else [x[b] for x in bounds])]
            if not keys:
                continue
            at, slot = table[b, np.array(keys) // page], np.array(keys) % page
            for h in range(H):
                k, v = (c[at, h // (H // heads), slot] for c in (k_cache, v_cache))
                s = k @ q[b, h, t] * scale
                top = s.max()
                p = np.exp(s - top)
                total = p.sum()
                out[b, h, t], mass[b, h, t] = p @ v / total, p @ np.abs(v) / total
                lse[b, h, t] = top + np.log(total)
                size[b, h, t] = (np.abs(k) @ np.abs(q[b, h, t])).max() * scale
    return out, lse, mass, size


def fork(pools, table, lens, parents, new_pages, page):
    """(pools, table, lens) after children took over from their parents."""
    pools = [np.array(p) for p in pools]
    rows = np.full((len(parents), table.shape[1]), -1, np.int32)
    out_lens = np.zeros(len(parents), np.int32)
    copies = []
    for r, (parent, fresh) in enumerate(zip(parents, new_pages)):
        if not 0 <= parent < len(lens):
            continue
        rows[r], out_lens[r] = table[parent], lens[parent]
        if fresh < 0:
            continue
        full, rest = divmod(max(int(lens[parent]), 0), page)
        rows[r, full:] = -1
        if rest and full < table.shape[1]:
            rows[r, full] = fresh
            copies.append((int(table[parent, full]), int(fresh)))
    for p in pools:
        old = p.copy()
        for source, to in copies:
            if 0 <= source < len(p) and 0 <= to < len(p):
                p[to] = old[source]
    return pools, rows, out_lens


def free_list(table, num_pages):
    used = {int(x) for x in np.ravel(table) if 0 <= x < num_pages}
    unused = [p for p in range(num_pages) if p not in used]
    return np.array(unused + [-1] * len(used), np.int32), len(unused)


def compact(pools, table):
    """(pools, table, used) with the used pages moved to the front."""
    pools = [np.array(p) for p in pools]
    num_pages = len(pools[0])
    used = sorted({int(x) for x in np.ravel(table) if 0 <= x < num_pages})
    behind = [p for p in used if p >= len(used)]
    holes = [p for p in range(len(used)) if p not in set(used)]
    to = dict(zip(behind, holes))
    for p in pools:
        for source, target in to.items():
            p[target] = p[source]
    return pools, np.vectorize(lambda x: to.get(int(x), x), otypes=[np.int32])(table), len(used)
