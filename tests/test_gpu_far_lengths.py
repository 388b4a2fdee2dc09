"""GPU: sequences said to be far longer than the table has places, up to the largest length: the weights of the keys that it has, and attention to
them."""
import numpy as np
import pytest

import test_gpu_cache_weights as cache_weights
import test_gpu_tree as tree
from keys_util import ints, values_of
from oracle import keys_oracle as orc
from serving_util import check, decode_bounds, f64

pytestmark = pytest.mark.gpu

LENS = [2 ** 30 + 90, 2 ** 31 - 1, 2 ** 30, 70]


@pytest.mark.parametrize("H,Hk,T", [(4, 4, 1), (4, 1, 3), (4, 1, 20), (2, 1, 70)])
@pytest.mark.parametrize("mask", ["none", "window", "bounds"])
def test_weights_of_a_cache(mask, H, Hk, T):
    p = cache_weights._problem(T, [112, 112, 112, 70], H, Hk, T, 64, 16, "bf16", "bf16", hide=False)
    p["lens"] = ints(LENS)
    if mask == "window":
        p["window"] = 2 ** 30 - 1       # the first sequence's last row sees keys from place 91 on
    elif mask == "bounds":              # some of the keys from some of the rows
        last = np.array(LENS)[:, None] - 1
        at = np.arange(112) + 0 * last
        p["bounds"] = (last - at % (T + 2), np.where(at % 3, last + at % 2, 2 ** 31 - 1), last - T + 0 * at, last - T + at % 4)
    cache_weights._run(p, 0.5)


@pytest.mark.parametrize("H,Hk,T", [(4, 4, 9), (4, 1, 20)])
@pytest.mark.parametrize("window", [0, 2 ** 30 - 1])
def test_trees(window, H, Hk, T):
    p = tree._problem(T, [112, 112, 112, 70], H, Hk, T, 64, 16, "bf16", "bf16")
    p["lens"], p["window"] = ints(LENS), window
    for name in ("k_cache", "v_cache"):
        p[name].nan_to_num_(0.0, 0.0, 0.0)      # what was hidden at the lengths of its making need not be now
    out, lse = tree._call(p)
    k, v = values_of(p)
    ref, ref_lse, mass, size = orc.decode_tree(f64(p["q"]), k, v, p["table"].cpu().numpy(), LENS, p["parents"], 0.125, window)
    bound, lse_bound = decode_bounds("bf16", ref, ref_lse, mass, size, 64, 112)
    some = ~np.isneginf(ref_lse)
    assert np.array_equal(np.isneginf(f64(lse)), ~some)
    check(f64(out), ref, bound, "out")
    check(f64(lse)[some], ref_lse[some], lse_bound[some], "lse")
