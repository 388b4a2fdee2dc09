"""flashmask_decode_workspace_bytes is 0 for exactly the shapes that flashmask_decode refuses."""
import ctypes
import struct

import pytest
import torch

import paper_2410_01359_amd as fm

SHAPE, WORKSPACE = -2, -4
P = 1 << 20   # an aligned address, never followed: every call on it is refused


def _code(B, H, Hk, T, d, packed, nbytes=256):
    """What flashmask_decode says with too little scratch; caches stored head by head or token by token."""
    page = 16
    row, head = (Hk * d, d) if packed else (d, page * d)
    cache = struct.pack("@PP6qPPP7i", P, P, *(page * Hk * d, head, row) * 2, 0, 0, P, 0, Hk, d, 4, page, B, 3)
    strides = (ctypes.c_int64 * 6)(*(H * T * d, T * d, d) * 2)
    return fm.load_library().flashmask_decode(cache, P, P, None, None, None, None, 0, 0, 0.1, P, P, 0, H, T, strides, P, nbytes, None)


@pytest.mark.parametrize("packed", [False, True])
@pytest.mark.parametrize("d", [64, 128])
def test_a_shape_with_scratch_is_accepted(d, packed):
    refused = accepted = 0
    for B in (1, 2, 700, 16000, 20000, 40000, 65535, 65536):
        for Hk in (1, 3, 256, 512, 1024, 16384, 16385):
            for group in (1, 5, 16):
                for T in (1, 2, 33, 256, 257):
                    size = fm.flashmask_decode_workspace_bytes(B, Hk * group, Hk, T, d)
                    for nbytes in (256, 1 << 40) if size == 0 else (256,):
                        code = _code(B, Hk * group, Hk, T, d, packed, nbytes)
                        assert code == (WORKSPACE if size else SHAPE), (B, Hk, group, T, size, code)
                    refused += size == 0
                    accepted += size > 0
    assert refused > 100 and accepted > 100


@pytest.mark.parametrize("packed", [False, True])
@pytest.mark.parametrize("B,Hk,group,T", [(65535, 1024, 1, 1), (65535, 16384, 1, 1), (16384, 16384, 1, 1), (65535, 512, 1, 33)])
def test_no_scratch_for_more_workgroups_than_any_call_may_have(B, Hk, group, T, packed):
    for d in (64, 128):
        assert fm.flashmask_decode_workspace_bytes(B, Hk * group, Hk, T, d) == 0
        assert _code(B, Hk * group, Hk, T, d, packed, 1 << 40) == SHAPE


@pytest.mark.gpu
def test_more_workgroups_than_a_launch_holds():
    """20000 sequences of 1024 heads that are not stored side by side; every hundredth one is the same."""
    B, same, heads, d = 20000, 100, 1024, 64
    gen = torch.Generator(device="cuda").manual_seed(1)
    cache = [torch.randn((4, heads, 16, d), device="cuda", generator=gen).bfloat16() for _ in range(2)]
    q = torch.randn((same, heads, 1, d), device="cuda", generator=gen).bfloat16()
    lens = torch.arange(same, device="cuda", dtype=torch.int32) % 19
    table = torch.randint(0, 4, (same, 2), device="cuda", generator=gen, dtype=torch.int32)
    want, want_lse = fm.flashmask_decode(q, *cache, table, lens, 0.125)
    out, lse = fm.flashmask_decode(q.repeat(B // same, 1, 1, 1), *cache, table.repeat(B // same, 1), lens.repeat(B // same), 0.125)
    assert (out.view(B // same, *want.shape) == want).all() and (lse.view(B // same, *want_lse.shape) == want_lse).all()
    assert want.isfinite().all() and want_lse[1:19].isfinite().all() and want_lse[0].isneginf().all()
