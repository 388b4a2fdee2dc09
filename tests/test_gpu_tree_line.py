"""GPU: flashmask_decode_tree on both sides of the lines between its two kernels, which differ with the cache's type and d: against the definition, with a workspace of
just the size that is asked for, which no type of cache writes beyond."""
import pytest
import torch

import test_gpu_tree as tree

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("type,cache", [("bf16", "bf16"), ("f16", "f16"), ("bf16", "e4m3"), ("f16", "e4m3")])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("H,Hk,T", [(1, 1, 47), (4, 2, 24), (8, 2, 12), (5, 1, 13), (2, 2, 63), (2, 2, 64), (16, 4, 19), (4, 1, 20), (79, 1, 1), (80, 1, 1)])
def test_both_sides_of_the_line(H, Hk, T, d, type, cache):
    import paper_2410_01359_amd as fm
    p = tree._problem(T, [900, 70, 0], H, Hk, T, d, 16, type, cache, mask="bounds" if T == 19 else "none")
    tree._check(p, type)
    want = tree._call(p)
    size = fm.flashmask_decode_tree_workspace_bytes(3, H, Hk, T, d)
    room = torch.full((size + (1 << 16),), 0xa5, dtype=torch.uint8, device="cuda")
    got = tree._call(p, workspace=room[:size])
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    assert (room[size:] == 0xa5).all()
    with pytest.raises(fm.FlashMaskError):
        tree._call(p, workspace=room[:256])
