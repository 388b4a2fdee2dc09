"""GPU: rows whose lse is -inf give the keys that they see no weight, whatever they and the keys hold: NaN, infinities, scores of either sign."""
import numpy as np
import pytest
import torch

import test_gpu_cache_weights as cache_weights
import test_gpu_weights as prompt
from keys_util import check_weights, ints, values_of
from oracle import cache_oracle, keys_oracle as orc
from serving_util import f64

pytestmark = pytest.mark.gpu

JUNK = (torch.nan, torch.inf, -torch.inf, 1e30)


def _silence(q, lse, which):
    """Rows `which` of q [.., rows, d], and lse [.., rows] with -inf there."""
    for n, i in enumerate(which):
        if n % 5 < 4:       # and some as they are
            q[..., i, :] = JUNK[n % 5]
            q[..., i, 1::2] *= -1
        lse[..., i] = -torch.inf


def _clean(x):
    return np.where(np.isfinite(x), x, 0)


@pytest.mark.parametrize("kind", ["full", "causal", "window", "docs"])
@pytest.mark.parametrize("N,d,which", [(333, 64, [332]), (333, 128, [0, 63, 64, 65, 200, 331, 332]), (700, 64, range(0, 700, 3)), (130, 64, range(130)), (1, 64, [0])])
def test_a_prompt(kind, N, d, which):
    import paper_2410_01359_amd as fm
    q, k, lse, bounds = prompt._problem(N, 2, 4, 2, N, d, kind)
    _silence(q[1], lse[1], which)
    if kind == "causal" and N - 1 in which:      # the last key is seen by the last row alone
        k[1, :, N - 1] = torch.nan
    got = fm.flashmask_weights(q, k, lse, *(ints(x) for x in bounds), d ** -0.5)
    check_weights(got, *orc.weights(_clean(f64(q)), _clean(f64(k)), f64(lse), bounds, d ** -0.5), d)
    if len(which) == N:
        assert (got[1] == 0).all()


@pytest.mark.parametrize("mask", ["none", "window", "bounds"])
@pytest.mark.parametrize("H,Hk,T,d", [(4, 4, 1, 64), (8, 2, 4, 128), (5, 1, 3, 64), (4, 1, 20, 64), (20, 1, 64, 64), (3, 1, 100, 128)])
@pytest.mark.parametrize("type,cache", [("bf16", "bf16"), ("f16", "e4m3")])
def test_a_cache(type, cache, H, Hk, T, d, mask):
    import paper_2410_01359_amd as fm
    lens = [200, 130, 70, 64]
    p = cache_weights._problem(T, lens, H, Hk, T, d, 16, type, cache, mask=mask, hide=False)
    k, _ = values_of(p)
    table, bounds = p["table"].cpu().numpy(), p["bounds"]
    lse = torch.tensor(cache_oracle.decode(f64(p["q"]), _clean(k), _clean(k), table, lens, d ** -0.5, p["window"], bounds)[1], dtype=torch.float32,
                       device="cuda")
    rows = [(h, t) for h in range(H) for t in range(T)]
    for b, some in ((0, rows[::3]), (1, rows[-1:]), (2, rows)):
        for n, (h, t) in enumerate(some):
            _silence(p["q"][b, h], lse[b, h], [t] if n % 2 else [])
            lse[b, h, t] = -torch.inf
    # the last key of the first sequence: seen by the last token alone, whose rows are silent here; all keys of the third
    lse[0, :, -1] = -torch.inf
    for b, j in [(0, 199)] + [(2, j) for j in range(70)]:
        page, slot = cache_oracle.place(table, len(p["k_cache"]), 16, b, j)
        p["k_cache"][page, :, slot] = torch.nan
    k = _clean(values_of(p)[0])
    before = torch.rand((4, Hk, 208), device="cuda")
    want = orc.cache_weights(_clean(f64(p["q"])), k, table, lens, f64(lse), d ** -0.5, f64(before), 0.5, np.zeros((4, Hk, 208)), p["window"], bounds)
    got = fm.flashmask_cache_weights(p["q"], p["k_cache"], p["v_cache"], p["table"], p["lens"], lse, d ** -0.5, before, decay=0.5, out=torch.zeros_like(before),
                                     bounds=None if bounds is None else tuple(ints(x) for x in bounds), window=p["window"], k_scale=p["k_scale"],
                                     v_scale=p["v_scale"])
    check_weights(got, want[0], want[1], want[2] + 2, d)
