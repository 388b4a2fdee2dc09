"""GPU: bounds of a cache's or a prompt's keys at the ends of 32 bits, in either pair: any number is a bound, and an interval that ends before it begins is
empty, however far before."""
import numpy as np
import pytest
import torch

import test_gpu_cache_weights as cache_weights
import test_gpu_tree as tree
import test_gpu_weights as prompt
from keys_util import ints, values_of
from oracle import cache_oracle, keys_oracle as orc
from serving_util import check, decode_bounds, f64

pytestmark = pytest.mark.gpu

LOW, HIGH = -2 ** 31, 2 ** 31 - 1
KINDS = ("ends_far_below", "begins_and_ends_far_below", "both_end_far_below", "pairs_exchanged", "far_above", "any")


def _bounds(kind, lens, T, N, seed):
    """(lts, lte, uts, ute) [sequences, N].  But for "any" they leave every row."""
    lens = np.maximum(np.asarray(lens), 0)[:, None]
    full = lambda x: np.broadcast_to(np.asarray(x, np.int64), (len(lens), N)).copy()
    zero, low, high, end = full(0), full(LOW), full(HIGH), full(lens)
    if kind == "ends_far_below":
        return zero, low, end, end
    if kind == "begins_and_ends_far_below":
        return low, low, end, end
    if kind == "both_end_far_below":
        return zero, low, end, low
    if kind == "pairs_exchanged":
        return end, end, zero, low
    if kind == "far_above":
        return high, low, end, high
    rng = np.random.default_rng(seed)
    ends = np.concatenate([full(x)[:, :, None] for x in (LOW, LOW + 1, -1, 0, lens - T, lens - 1, lens, N, HIGH - 1, HIGH)], 2)
    return tuple(np.take_along_axis(ends, rng.integers(0, ends.shape[2], (len(lens), N, 1)), 2)[:, :, 0] for _ in range(4))


@pytest.mark.parametrize("lens,H,Hk,T,d,page", [([200, 65, 3, 0], 4, 4, 1, 64, 16), ([150, 70], 4, 1, 4, 128, 32), ([130, 64], 12, 2, 7, 64, 16),
                                                ([200, 90], 2, 1, 100, 64, 16)])
@pytest.mark.parametrize("kind", KINDS)
def test_weights_of_a_cache(kind, lens, H, Hk, T, d, page):
    p = cache_weights._problem(T, lens, H, Hk, T, d, page, "bf16", "bf16", hide=False)
    p["bounds"] = _bounds(kind, lens, T, p["table"].shape[1] * page, T)
    cache_weights._run(p, 0.5)


@pytest.mark.parametrize("lens,H,Hk,T,d,page", [([200, 65, 0], 4, 4, 9, 64, 16), ([300, 70], 3, 1, 21, 128, 32), ([200, 333, 40], 8, 2, 16, 64, 16),
                                                ([300, 90], 2, 1, 70, 128, 32)])
@pytest.mark.parametrize("shape", ["chain", "tree"])
@pytest.mark.parametrize("kind", KINDS)
def test_trees(kind, shape, lens, H, Hk, T, d, page):
    """On both sides of 64 query rows to a K/V head."""
    p = tree._problem(T, lens, H, Hk, T, d, page, "bf16", "bf16", kind=shape)
    p["np_bounds"] = _bounds(kind, lens, T, p["table"].shape[1] * page, T)
    tree._check(p, "bf16")


@pytest.mark.parametrize("kind", KINDS)
def test_weights_of_a_prompt(kind):
    N, d = 333, 64
    q, k, _, _ = prompt._problem(4, 1, 4, 2, N, d, "full")
    bounds = _bounds(kind, [N], N, N, 4)
    seen = np.array([[not orc.hidden([x[0] for x in bounds], i, j) for j in range(N)] for i in range(N)])
    s = np.where(seen, f64(q)[0] @ f64(k)[0].repeat(2, 0).transpose(0, 2, 1) * d ** -0.5, -np.inf)
    with np.errstate(divide="ignore"):
        lse = np.log(np.exp(s).sum(2))[None]
    prompt._check((q, k, torch.tensor(lse, dtype=torch.float32, device="cuda"), bounds))


@pytest.mark.parametrize("H,T", [(4, 1), (4, 20)])
@pytest.mark.parametrize("kind", KINDS)
def test_decoding_of_one_and_many_new_tokens(kind, H, T):
    import paper_2410_01359_amd as fm
    p = cache_weights._problem(50 + T, [200, 65, 0], H, 1, T, 64, 16, "bf16", "bf16", hide=False)
    bounds = _bounds(kind, [200, 65, 0], T, p["table"].shape[1] * 16, T)
    out, lse = fm.flashmask_decode(p["q"], p["k_cache"], p["v_cache"], p["table"], p["lens"], 0.125, bounds=tuple(ints(x) for x in bounds))
    k, v = (np.where(np.isfinite(x), x, 0) for x in values_of(p))
    ref, ref_lse, mass, size = cache_oracle.decode(f64(p["q"]), k, v, p["table"].cpu().numpy(), [200, 65, 0], 0.125, 0, bounds)
    bound, lse_bound = decode_bounds("bf16", ref, ref_lse, mass, size, 64, 200)
    some = ~np.isneginf(ref_lse)
    assert np.array_equal(np.isneginf(f64(lse)), ~some)
    check(f64(out), ref, bound, "out")
    check(f64(lse)[some], ref_lse[some], lse_bound[some], "lse")
