"""Numbers that do not fit the C ABI's 32-bit ints are refused by the binding, or mean what they say, instead of losing their upper bits."""
import numpy as np
import pytest
import torch

import paper_2410_01359_amd as fm

BEYOND = 1 << 32


def test_sizes_of_scratch():
    assert fm.flashmask_cache_plan_bytes(100) > 0 and fm.flashmask_decode_workspace_bytes(2, 8, 2, 1, 64) > 0
    assert fm.flashmask_cache_plan_bytes(BEYOND + 100) == 0 and fm.flashmask_cache_plan_bytes(100 - BEYOND) == 0
    for at in range(5):
        shape = [2, 8, 2, 1, 64]
        for far in (BEYOND, -BEYOND):
            shape[at] += far
            assert fm.flashmask_decode_workspace_bytes(*shape) == 0
            shape[at] -= far


def _ints(x):
    return torch.tensor(np.asarray(x), dtype=torch.int32, device="cuda")


@pytest.mark.gpu
def test_windows_of_any_size():
    """A window beyond every length hides nothing."""
    gen = torch.Generator(device="cuda").manual_seed(1)
    cache = [torch.randn((8, 2, 16, 64), device="cuda", generator=gen).bfloat16() for _ in range(2)]
    q = torch.randn((1, 4, 2, 64), device="cuda", generator=gen).bfloat16()
    args = (q, *cache, _ints([range(8)]), _ints([125]), 0.125)
    want = fm.flashmask_decode(*args)
    assert not torch.equal(fm.flashmask_decode(*args, window=5)[0], want[0])
    for window in (125, (1 << 30) - 1, 1 << 30, (1 << 31) - 1, 1 << 31, BEYOND, BEYOND + 5, 1 << 70):
        got = fm.flashmask_decode(*args, window=window)
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1]), window
    for window in (-1, -BEYOND, 5 - BEYOND):
        with pytest.raises(fm.FlashMaskError):
            fm.flashmask_decode(*args, window=window)


@pytest.mark.gpu
def test_pages_and_layouts_beyond_32_bits():
    pool = torch.zeros((4, 2, 16, 64), device="cuda", dtype=torch.bfloat16)
    table, one = _ints([[0, 1]]), _ints([0])
    q = torch.ones((1, 2, 3, 64), device="cuda", dtype=torch.bfloat16)
    freqs = torch.ones(32, device="cuda", dtype=torch.float64)
    token, at = torch.ones((1, 2, 64), device="cuda", dtype=torch.bfloat16), _ints([3])
    for far in (BEYOND, -BEYOND):
        for call in (lambda: fm.flashmask_cache_fork([pool], table, one, one, one, 16 + far),
                     lambda: fm.flashmask_rope(q, q, freqs, layout=far), lambda: fm.flashmask_rope_bwd(q, q, freqs, layout=far + 1),
                     lambda: fm.flashmask_cache_append(token, token, pool, pool.clone(), table, one, at, freqs=freqs, layout=far),
                     lambda: fm.flashmask_cache_free_list(table, far + 4)):
            with pytest.raises(fm.FlashMaskError):
                call()
    torch.cuda.synchronize()
