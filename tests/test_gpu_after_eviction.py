"""GPU: the calls over the cache after an eviction count rows, windows and bounds by place: what they give is what they give over a cache that was only ever
written the kept tokens."""
import numpy as np
import pytest
import torch

from keys_util import ints, paged, queries, spare_pages, values_of
from oracle import cache_oracle
from serving_util import check, decode_bounds, f64

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("shared", [True, False])
@pytest.mark.parametrize("window", [0, 20])
def test_decoding_after_an_eviction(window, shared):
    import paper_2410_01359_amd as fm
    lens, H, Hk, d, page, keep, T = [200, 90, 30], 4, 2, 64, 16, 48, 3
    p = paged(3, lens, Hk, page, d, "bf16", spare=9)
    new_table = ints(spare_pages(p)[:9].reshape(3, 3))
    gen = torch.Generator(device="cuda").manual_seed(1)
    weights = torch.rand((3, 1 if shared else Hk, 208), device="cuda", generator=gen)
    k, v = values_of(p)
    table, left, _, kept = fm.flashmask_cache_evict(p["k_cache"], p["v_cache"], p["table"], p["lens"], weights, new_table, keep, first=2, recent=10)
    assert left.tolist() == [48, 48, 30]
    # the kept tokens' keys and values, place after place, as a cache of one page to a sequence
    old, kept = p["table"].cpu().numpy(), kept.cpu().numpy()
    plain = np.zeros((2, 3, Hk, keep, d))
    for b in range(3):
        for h in range(Hk):
            for i, j in enumerate(kept[b, 0 if shared else h]):
                if j >= 0:
                    at = cache_oracle.place(old, k.shape[0], page, b, int(j))
                    plain[:, b, h, i] = k[at[0], h, at[1]], v[at[0], h, at[1]]
    # bounds by place, of rows counted by place: every third key of the kept ones is hidden from the second new token
    bounds = None
    if shared:
        at, rows = np.arange(keep) + np.zeros((3, 1), int), left.cpu().numpy()[:, None] - T
        bounds = (np.where(at % 3 == 0, rows + 1, 0), np.where(at % 3 == 0, rows + 2, 0), 0 * at, 0 * at)
    q = queries(3, 3, H, T, d, "bf16")
    out, lse = fm.flashmask_decode(q, p["k_cache"], p["v_cache"], table, left, d ** -0.5, window=window,
                                   bounds=None if bounds is None else tuple(ints(x) for x in bounds))
    ref, ref_lse, mass, size = cache_oracle.decode(f64(q), plain[0], plain[1], np.arange(3)[:, None], [48, 48, 30], d ** -0.5, window, bounds)
    bound, lse_bound = decode_bounds("bf16", ref, ref_lse, mass, size, d, keep)
    check(f64(out), ref, bound, "out")
    check(f64(lse), ref_lse, lse_bound, "lse")
