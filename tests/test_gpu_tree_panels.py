"""GPU: flashmask_decode_tree where a chunk of a sequence is longer than the 4096 keys that are looked over at a time: every such panel with tiles that all
rows see whole and tiles that take the element mask, and what is carried from one to the next."""
import numpy as np
import pytest
import torch

from keys_util import ints
from oracle import keys_oracle as orc
from serving_util import TYPES, check, decode_bounds, f64

pytestmark = pytest.mark.gpu

HEADS, T, PAGE = 260, 64, 64        # so many workgroups to a chunk of keys that a sequence is one chunk
LEN = 9001
SOME = (0, 1, 131, 259)


def _problem(type, cache, d, mask):
    gen = torch.Generator(device="cuda").manual_seed(d)
    rng = np.random.default_rng(d)
    columns = -(-LEN // PAGE)
    pages = columns + 2
    p = {"type": type, "d": d, "q": torch.randn((1, HEADS, T, d), device="cuda", generator=gen).to(TYPES[type])}
    for name in ("k", "v"):
        p[name] = torch.randn((pages, HEADS, PAGE, d), device="cuda", generator=gen).to(TYPES[cache])
    table = rng.permutation(pages)[:columns]
    table[[3, 70, 100, 135]] = -1, pages, -5, 10 ** 6       # a hole in each panel, two in the second; the third begins at page 128
    p["table"], p["parents"] = table, np.maximum(np.arange(T) - rng.integers(1, 7, T), -1)
    p["scales"] = [torch.rand(HEADS, device="cuda", generator=gen) + 0.5 for _ in range(2)] if cache == "e4m3" else [None, None]
    start = LEN - T
    lines = orc.ancestors(p["parents"])
    depth = np.array([len(x) - 1 for x in lines])
    row, j = (start + depth)[:, None], np.arange(LEN)
    seen = np.zeros((T, LEN), bool)
    seen[:, :start] = True
    for t, line in enumerate(lines):
        seen[t, [start + u for u in line]] = True
    p["window"] = {"window": 8000, "inner": 3}.get(mask, 0)     # the first ends inside the first panel
    if p["window"]:
        at = np.append(j[:start], start + depth)
        seen &= at > row - p["window"]
    p["bounds"] = None
    if mask == "bounds":        # some tiles that nobody sees, some that some rows do
        lts = np.full(LEN, LEN)
        lts[200:500], lts[4500:4700], lts[8300:8400] = start, start + 3, 0
        lte, uts, ute = np.full(LEN, LEN), np.zeros(LEN, int), np.zeros(LEN, int)
        uts[::777], ute[::777] = start + 1, start + 5
        p["bounds"] = np.stack([lts, lte, uts, ute])
        seen &= ~(((lts <= row) & (row < lte)) | ((uts <= row) & (row < ute)))
    there = (table >= 0) & (table < pages)
    p["seen"] = seen & there[j // PAGE]
    # what no row sees is no number
    for at in np.nonzero(~seen.any(0) & there[j // PAGE])[0]:
        for name in ("k", "v"):
            p[name][int(table[at // PAGE]), :, at % PAGE] = torch.nan
    return p


def _call(p):
    import paper_2410_01359_amd as fm
    bounds = None if p["bounds"] is None else tuple(ints(x[None]) for x in p["bounds"])
    return fm.flashmask_decode_tree(p["q"], p["k"], p["v"], ints(p["table"][None]), ints([LEN]), ints(p["parents"][None]), p["d"] ** -0.5, bounds=bounds,
                                    window=p["window"], k_scale=p["scales"][0], v_scale=p["scales"][1])


def _reference(p, h):
    """out, lse, sum of p |v|, largest scale * sum |q||k| of head h, in 64 bits."""
    seen = torch.tensor(p["seen"], device="cuda")
    pages = torch.tensor(np.where((p["table"] >= 0) & (p["table"] < len(p["k"])), p["table"], 0), device="cuda")
    rows = [x[pages, h].double().flatten(0, 1)[:LEN] * (1.0 if s is None else s[h].double()) for x, s in zip((p["k"], p["v"]), p["scales"])]
    k, v = (x.nan_to_num(0.0) for x in rows)
    q, scale = p["q"][0, h].double(), p["d"] ** -0.5
    s = torch.where(seen, q @ k.T * scale, -torch.inf)
    lse = s.logsumexp(1)
    w = (s - lse[:, None]).exp()
    return [f64(x) if x.dtype != torch.float64 else x.cpu().numpy()
            for x in (w @ v, lse, w @ v.abs(), (q.abs() @ k.abs().T * seen).amax(1) * scale)]


@pytest.mark.parametrize("mask", ["none", "window", "inner", "bounds"])
@pytest.mark.parametrize("type,cache,d", [("bf16", "bf16", 64), ("f16", "f16", 128), ("bf16", "e4m3", 64), ("f16", "e4m3", 128)])
def test_against_the_definition(type, cache, d, mask):
    p = _problem(type, cache, d, mask)
    out, lse = _call(p)
    assert torch.isfinite(out).all() and torch.isfinite(lse).all()
    for h in SOME:
        ref, ref_lse, mass, size = _reference(p, h)
        bound, lse_bound = decode_bounds(type, ref, ref_lse, mass, size, d, LEN)
        check(f64(out[0, h]), ref, bound, f"head {h} out")
        check(f64(lse[0, h]), ref_lse, lse_bound, f"head {h} lse")


@pytest.mark.parametrize("mask", ["none", "bounds"])
@pytest.mark.parametrize("type,cache,d", [("bf16", "bf16", 128), ("f16", "e4m3", 64), ("bf16", "e4m3", 128)])
def test_odd_values_reach_those_that_see_them(type, cache, d, mask):
    """NaN in elements of their own of keys of all panels: in tiles with a hole, in tiles that only some rows see, among the drafted tokens."""
    p = _problem(type, cache, d, mask)
    start, elements = LEN - T, {}
    for n, at in enumerate((5, 3 * PAGE + 70, 777 * 2, 4600, 4650, 71 * PAGE + 3, 101 * PAGE, 777 * 11, 134 * PAGE + 63, start + 1, LEN - 1)):
        page = int(p["table"][at // PAGE])
        assert 0 <= page < p["v"].shape[0]
        p["v"][page, :, at % PAGE, 2 * n] = torch.nan
        elements[2 * n] = at
    out = f64(_call(p)[0])[0]
    for element in range(d):
        at = elements.get(element)
        want = p["seen"][:, at] if at is not None else np.zeros(T, bool)
        assert np.array_equal(np.isnan(out[:, :, element]), np.broadcast_to(want, (HEADS, T))), (element, at)
