"""Shared by the GPU tests of the cache operators: paged caches with junk wherever nothing is cached, and bounds on rounding errors."""
import numpy as np
import torch

from oracle import cache_oracle as orc

TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32, "e4m3": torch.float8_e4m3fn}
# the smallest value above 0 of each type
TINY = {"bf16": 2.0 ** -133, "f16": 2.0 ** -24, "f32": 2.0 ** -149, "e4m3": 2.0 ** -9}


def f64(t):
    return t.detach().float().cpu().numpy().astype(np.float64)


def rounding(type, x):
    """Half a step of the type at |x|."""
    return torch.finfo(TYPES[type]).eps / 2 * np.abs(x) + TINY[type] / 2


def strided(t, packed):
    """The tensor as a view of one that is stored with its axes 1 and 2 exchanged."""
    return t.transpose(1, 2).contiguous().transpose(1, 2) if packed else t.contiguous()


def cache_of(gen, type, pages, heads, page, d, packed=False, junk=False):
    """Pages [pages, heads, page, d] of normal values, or of NaN and infinities."""
    x = torch.randn((pages, heads, page, d), device="cuda", generator=gen)
    if junk:
        x = torch.where(x > 0.5, torch.inf, torch.where(x < -0.5, -torch.inf, torch.nan))
        if type == "e4m3":
            x = torch.full_like(x, torch.nan)   # no infinities
    return strided(x.to(TYPES[type]), packed)


def rows_of(cache, table, lens):
    """Index (page, slot) of every cached token."""
    page, pages = cache.shape[2], cache.shape[0]
    at = [(int(table[b, j // page]), j % page) for b in range(table.shape[0]) for j in range(min(int(lens[b]), table.shape[1] * page))
          if 0 <= table[b, j // page] < pages]
    return tuple(torch.tensor(x, dtype=torch.long, device="cuda") for x in zip(*at)) if at else None


def raw(t):
    return t.view(torch.uint8) if t.element_size() == 1 else t.view(torch.int16) if t.element_size() == 2 else t


def decode_bounds(type, ref, lse, mass, size, d, keys):
    """Bounds on the errors of flashmask_decode's out and lse (arrays of the fp64 result, its sum of p |v|, the largest scale * sum |q||k| and
    the number of keys at most).  A score's d products are added in 32 bits; its exponent is one rounding of a number as large as the
    score, twice; sums of p over at most keys / 16 additions and a few joins; the probabilities enter the second product with 16 bits
    (bf16) or 22 (f16), f16's no finer than half its smallest value; out is rounded once."""
    step = 2.0 ** -23
    score = (d + 8) * step * size + 2 * step * (np.abs(np.where(np.isfinite(lse), lse, 0)) + size) + 4 * step
    sums = (keys / 16 + 64) * step
    p = 2.0 ** -17 if type == "bf16" else 2.0 ** -22
    tiny = 0 if type == "bf16" else 2.0 ** -25 * keys
    relative = (2 * score + 2 * sums + p)[..., None]
    out = rounding(type, ref) + (relative + tiny) * (mass + np.abs(ref)) * 1.01 + tiny * np.abs(mass).max(initial=0.0)
    return out, score + sums + 2.0 ** -21


def check(got, ref, bound, what):
    got = np.asarray(got, np.float64)
    assert np.isfinite(got).all(), f"{what}: not finite"
    excess = np.abs(got - ref) - bound
    if not excess.size:
        return
    at = np.unravel_index(np.argmax(excess), excess.shape)
    assert excess[at] <= 0, f"{what}{list(at)}: {got[at]} for {ref[at]}, bound {np.broadcast_to(bound, ref.shape)[at]:.3g}"


__all__ = ["TYPES", "TINY", "f64", "rounding", "strided", "cache_of", "rows_of", "raw", "decode_bounds", "check", "orc"]
