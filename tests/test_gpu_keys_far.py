"""GPU: the operators on weights, eviction and trees where pages and rows lie more than 2^32 bytes into their memory: the same bits as of the same
tokens near its begin."""
import numpy as np
import pytest
import torch

from keys_util import ints, paged, queries

pytestmark = pytest.mark.gpu
FAR = (5 << 30) // (2 * 16 * 64 * 2)      # pages of 2 heads, 16 tokens and 64 elements of 16 bits in 5 GiB


@pytest.fixture(scope="module")
def pools():
    return [torch.empty((FAR, 2, 16, 64), dtype=torch.bfloat16, device="cuda") for _ in range(2)]


def _both(seed, lens, pools):
    """The problem with its own pools, and with its pages moved to the ends of large ones."""
    near = paged(seed, lens, 2, 16, 64, "bf16", spare=40)
    n = near["k_cache"].shape[0]
    for pool, c in zip(pools, (near["k_cache"], near["v_cache"])):
        pool[-n:] = c
    table = near["table"]
    return near, {**near, "k_cache": pools[0], "v_cache": pools[1], "table": torch.where(table >= 0, table + (FAR - n), table)}, n


def _decode(p, q, T, seed):
    import paper_2410_01359_amd as fm
    parents = ints([[t - 1 if t % 3 else t // 2 - 1 for t in range(T)] for _ in range(len(p["lens"]))])
    return fm.flashmask_decode_tree(q, p["k_cache"], p["v_cache"], p["table"], p["lens"], parents, 0.125)


@pytest.mark.parametrize("T", [5, 50])
def test_trees_and_weights(T, pools):
    import paper_2410_01359_amd as fm
    near, far, _ = _both(1, [700, 64, 90], pools)
    q = queries(1, 3, 8, T, 64, "bf16")
    a, b = (_decode(p, q, T, 1) for p in (near, far))
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    a, b = (fm.flashmask_cache_weights(q, p["k_cache"], p["v_cache"], p["table"], p["lens"], a[1], 0.125) for p in (near, far))
    assert torch.equal(a, b) and torch.isfinite(a).all()


def test_eviction_and_accepted_paths(pools):
    import paper_2410_01359_amd as fm
    near, far, n = _both(2, [300, 64, 90], pools)
    weights = torch.rand((3, 2, 304), device="cuda", generator=torch.Generator(device="cuda").manual_seed(1))
    fresh = np.setdiff1d(np.arange(n), near["table"].cpu().numpy())[:15].reshape(3, 5)
    after = []
    for p, first in ((near, 0), (far, FAR - n)):
        table, lens, _, kept = fm.flashmask_cache_evict(p["k_cache"], p["v_cache"], p["table"], p["lens"], weights, ints(fresh + first), 70, first=3,
                                                        recent=20)
        lens = fm.flashmask_cache_accept([p["k_cache"], p["v_cache"]], table, lens, 10, ints([[1, 4, 5, -1], [0, 1, -1, -1], [9, -1, -1, -1]]))
        after.append((torch.where(table >= 0, table - first, table), lens, kept))
    assert all(torch.equal(a, b) for a, b in zip(*after))
    for pool, c in zip(pools, (near["k_cache"], near["v_cache"])):
        assert torch.equal(pool[-n:].view(torch.int16), c.view(torch.int16))


def test_prompts():
    import paper_2410_01359_amd as fm
    space = torch.empty((2, (5 << 30) // 2), dtype=torch.bfloat16, device="cuda")     # batches 5 GiB apart
    N = 200
    q, k = (space[:, at:at + h * N * 64].view(2, h, N, 64) for at, h in ((0, 4), ((4 << 30) // 2, 2)))
    gen = torch.Generator(device="cuda").manual_seed(3)
    for x in (q, k):
        x.copy_(torch.randn(x.shape, device="cuda", generator=gen))
    at = torch.arange(N, dtype=torch.int32, device="cuda").repeat(2, 1)
    bounds = (torch.full_like(at, N), torch.full_like(at, N), torch.zeros_like(at), at)
    lse = torch.randn((2, 4, N), device="cuda", generator=gen) + 5
    assert torch.equal(fm.flashmask_weights(q, k, lse, *bounds, 0.125), fm.flashmask_weights(q.contiguous(), k.contiguous(), lse, *bounds, 0.125))
