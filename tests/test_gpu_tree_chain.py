"""GPU: a tree that is a chain is flashmask_decode, on both sides of 64 query rows to a K/V head: outputs within what both may be off, lse within 32 bits of it."""
import numpy as np
import pytest

import test_gpu_tree as tree
from keys_util import ints, values_of
from oracle import cache_oracle
from serving_util import check, decode_bounds, f64

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("type,cache", [("bf16", "bf16"), ("f16", "e4m3")])
@pytest.mark.parametrize("mask", ["none", "window", "bounds"])
@pytest.mark.parametrize("lens,H,Hk,T,d", [([900, 33], 4, 2, 4, 128), ([700, 63, 20], 2, 2, 63, 64), ([900, 70], 8, 2, 16, 128), ([1300, 63, 9], 4, 1, 63, 64),
                                           ([500, 300], 1, 1, 252, 128)])
def test_a_chain_is_flashmask_decode(lens, H, Hk, T, d, mask, type, cache):
    import paper_2410_01359_amd as fm
    p = tree._problem(T, lens, H, Hk, T, d, 16, type, cache, mask=mask, kind="chain")
    bounds = None if p["np_bounds"] is None else tuple(ints(x) for x in p["np_bounds"])
    out, lse = (f64(x) for x in tree._call(p))
    want, want_lse = (f64(x) for x in fm.flashmask_decode(p["q"], p["k_cache"], p["v_cache"], p["table"], p["lens"], p["scale"], bounds=bounds,
                                                          window=p["window"], k_scale=p["k_scale"], v_scale=p["v_scale"]))
    k, v = (np.where(np.isfinite(x), x, 0) for x in values_of(p))       # what no row sees is no number
    ref, ref_lse, mass, size = cache_oracle.decode(f64(p["q"]), k, v, p["table"].cpu().numpy(), lens, p["scale"], p["window"], p["np_bounds"])
    bound, lse_bound = decode_bounds(type, ref, ref_lse, mass, size, d, max(lens))
    some = ~np.isneginf(ref_lse)
    assert np.array_equal(np.isneginf(lse), ~some) and np.array_equal(np.isneginf(want_lse), ~some)
    # each is within its bound of the definition, so that they are within twice that of each other
    check(out, want, 2 * bound, "out")
    check(lse[some], want_lse[some], 2 * lse_bound[some], "lse")
    assert lse_bound[some].max() < 1e-3
