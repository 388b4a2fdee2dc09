"""Rotary positions, the paged key-value cache and attention of new tokens over it (see include/flashmask.h for the contract).

Argument marshalling only, as in binding.py: every step runs in the HIP kernels, and nothing falls back.  A cache is a pair of
tensors indexed [pages, heads, tokens of a page, d] (any strides, d contiguous), a page table int32 [sequences, columns] with -1
where there is no page, and for 8-bit caches (torch.float8_e4m3fn) a scale for each head.
"""
from __future__ import annotations

import ctypes
import struct

import torch

from .binding import FlashMaskError, _check, _dev, _stream, load_library

FM_ROPE_HALF, FM_ROPE_INTERLEAVED = 0, 1

_TYPE = {torch.bfloat16: 0, torch.float16: 1, torch.float32: 2, torch.float8_e4m3fn: 3}
_CACHE = struct.Struct("@PP6qPPP7i")   # flashmask_cache
_HERE = torch.cuda.current_device


def _index(t, shape, name: str) -> int:
    """Address of an int32 tensor of this shape."""
    if not (t.is_cuda and t.dtype is torch.int32 and t.is_contiguous()):
        _dev(t, torch.int32, name)
    if t.shape != shape:
        raise FlashMaskError(f"{name} must be {list(shape)}, got {list(t.shape)}")
    return t.data_ptr()


def _data(t, dims: int, name: str, types=(torch.bfloat16, torch.float16)):
    """Element strides of a tensor of rows of d elements."""
    if not t.is_cuda:
        raise FlashMaskError(f"{name} must live on the GPU")
    if t.dtype not in types:
        raise FlashMaskError(f"{name} must be one of {types}, got {t.dtype}")
    strides = t.stride()
    if len(strides) != dims or strides[-1] != 1:
        raise FlashMaskError(f"{name} must have {dims} dimensions, the last one contiguous")
    return strides[:-1]


def _same_device(first, *others):
    device = first.get_device()
    if device != _HERE():
        raise FlashMaskError(f"the tensors are on GPU {device}, the current one is {_HERE()}")
    for t in others:
        if t is not None and t.get_device() != device:
            raise FlashMaskError("the tensors must be on one GPU")


def _vector(t, n: int, dtype, name: str) -> int:
    """Address of a vector; 0 for None."""
    if t is None:
        return 0
    if not (t.is_cuda and t.dtype is dtype and t.is_contiguous()):
        _dev(t, dtype, name)
    if t.dim() != 1 or t.shape[0] != n and (n >= 0 or t.shape[0] == 0):
        raise FlashMaskError(f"{name} must be a vector of {n} values" if n >= 0 else f"{name} must be a vector of some values")
    return t.data_ptr()


def _rope(entry: str, q, k, freqs, positions, layout, amp):
    types = (torch.bfloat16, torch.float16, torch.float32)
    sq, sk = _data(q, 4, "q", types), _data(k, 4, "k", types)
    B, H, N, d = q.shape
    Hk = k.shape[1]
    if k.dtype is not q.dtype or k.shape != (B, Hk, N, d):
        raise FlashMaskError("k must be [B,H_kv,N,d] of q's type and sizes")
    at = 0 if positions is None else _index(positions, (B, N), "positions")
    frequencies = _vector(freqs, -1, torch.float64, "freqs")
    _same_device(q, k, freqs, positions)
    q_out, k_out = torch.empty_like(q), torch.empty_like(k)
    strides = (ctypes.c_int64 * 12)(*sq, *sk, *q_out.stride()[:3], *k_out.stride()[:3])
    _check(getattr(load_library(), entry)(q.data_ptr(), k.data_ptr(), q_out.data_ptr(), k_out.data_ptr(), frequencies, at,
                                          _TYPE[q.dtype], layout, amp, B, H, Hk, N, d, 2 * freqs.shape[0], strides, _stream()), entry)
    return q_out, k_out


def flashmask_rope(q, k, freqs, positions=None, *, layout: int = FM_ROPE_HALF, amp: float = 1.0):
    """q [B,H,N,d] and k [B,H_kv,N,d] (bf16, fp16 or fp32; any strides, d contiguous) with their first 2 * len(freqs) elements
    turned by the angles positions * freqs (positions int32 [B,N], None: 0..N-1; freqs float64).  Laid out like q and k."""
    return _rope("flashmask_rope", q, k, freqs, positions, layout, amp)


def flashmask_rope_bwd(dq, dk, freqs, positions=None, *, layout: int = FM_ROPE_HALF, amp: float = 1.0):
    """The gradients of flashmask_rope's results to those of its q and k."""
    return _rope("flashmask_rope_bwd", dq, dk, freqs, positions, layout, amp)


def _cache(k_cache, v_cache, table, k_scale, v_scale):
    """flashmask_cache as bytes, and [heads, page, d]."""
    types = (torch.bfloat16, torch.float16, torch.float8_e4m3fn)
    sk, sv = _data(k_cache, 4, "k_cache", types), _data(v_cache, 4, "v_cache", types)
    pages, heads, page, d = k_cache.shape
    if v_cache.shape != k_cache.shape or v_cache.dtype is not k_cache.dtype:
        raise FlashMaskError("k_cache and v_cache must have one shape and type")
    if table.dim() != 2:
        raise FlashMaskError("table must be [sequences, columns]")
    sequences, columns = table.shape
    where = _index(table, table.shape, "table")
    scales = [_vector(s, heads, torch.float32, n) for s, n in ((k_scale, "k_scale"), (v_scale, "v_scale"))]
    return (_CACHE.pack(k_cache.data_ptr(), v_cache.data_ptr(), *sk, *sv, *scales, where, _TYPE[k_cache.dtype], heads, d, pages, page,
                        sequences, columns), heads, page, d)


def flashmask_cache_append(k, v, k_cache, v_cache, table, seqs, positions, *, q=None, freqs=None, layout: int = FM_ROPE_HALF,
                           amp: float = 1.0, k_scale=None, v_scale=None):
    """Write new tokens' keys (rotated where freqs is given) and values [tokens, H_kv, d] to the cache: token n goes to position
    positions[n] of sequence seqs[n] (outside the table's sequences: padding).  Returns the queries q [tokens, H, d], rotated, or
    None."""
    cache, heads, _, d = _cache(k_cache, v_cache, table, k_scale, v_scale)
    sk, sv = _data(k, 3, "k"), _data(v, 3, "v")
    n = k.shape[0]
    if k.shape != (n, heads, d) or v.shape != k.shape or v.dtype is not k.dtype:
        raise FlashMaskError("k and v must be [tokens, H_kv, d] of one type, heads and d those of the cache")
    seqs_at, positions_at = _index(seqs, (n,), "seqs"), _index(positions, (n,), "positions")
    frequencies = _vector(freqs, -1, torch.float64, "freqs")
    H, q_at, out_at, q_out, sq, so = 0, 0, 0, None, (0, 0), (0, 0)
    if q is not None:
        sq = _data(q, 3, "q")
        H = q.shape[1]
        if q.shape != (n, H, d) or q.dtype is not k.dtype:
            raise FlashMaskError("q must be [tokens, H, d] of k's type")
        if freqs is None:
            raise FlashMaskError("q is only rotated: it needs freqs")
    _same_device(k, v, k_cache, v_cache, table, seqs, positions, q, freqs, k_scale, v_scale)
    if n == 0:
        return None if q is None else torch.empty_like(q)
    if q is not None:
        q_out = torch.empty((n, H, d), dtype=q.dtype, device=q.device)
        q_at, out_at, so = q.data_ptr(), q_out.data_ptr(), (H * d, d)
    strides = (ctypes.c_int64 * 12)(0, sq[1], sq[0], 0, sk[1], sk[0], 0, sv[1], sv[0], 0, so[1], so[0])
    _check(load_library().flashmask_cache_append(cache, q_at, k.data_ptr(), v.data_ptr(), out_at, seqs_at, positions_at, frequencies,
                                                 _TYPE[k.dtype], layout, amp, n, H, 0 if freqs is None else 2 * freqs.shape[0], strides,
                                                 _stream()), "flashmask_cache_append")
    return q_out


def flashmask_decode_workspace_bytes(sequences: int, H: int, H_kv: int, T: int, d: int) -> int:
    return int(load_library().flashmask_decode_workspace_bytes(sequences, H, H_kv, T, d))


def flashmask_decode(q, k_cache, v_cache, table, lens, scale: float, *, bounds=None, window: int = 0, k_scale=None, v_scale=None,
                     workspace: torch.Tensor | None = None):
    """Attention of the last T tokens of every sequence, q [sequences, H, T, d], over the cache, which holds lens[b] tokens of
    sequence b, the new ones among them.  bounds: (lts, lte, uts, ute), int32 [sequences, columns]; window: keys that a row sees,
    itself among them (0: all).  Returns out (laid out like q) and lse (fp32 [sequences, H, T])."""
    cache, heads, _, d = _cache(k_cache, v_cache, table, k_scale, v_scale)
    sq = _data(q, 4, "q")
    B, H, T, d_q = q.shape
    if d_q != d or B != table.shape[0]:
        raise FlashMaskError("q must be [sequences, H, T, d] of the table's sequences and the cache's d")
    lens_at = _index(lens, (B,), "lens")
    lts = lte = uts = ute = None
    at, columns = (0, 0, 0, 0), 0
    if bounds is not None:
        if len(bounds) != 4 or bounds[0].numel() == 0:
            raise FlashMaskError("bounds must be (lts, lte, uts, ute), int32 [sequences, columns]")
        lts, lte, uts, ute = bounds
        columns = lts.shape[-1]
        at = [_index(x, (B, columns), n) for x, n in zip(bounds, ("lts", "lte", "uts", "ute"))]
    _same_device(q, k_cache, v_cache, table, lens, lts, lte, uts, ute, k_scale, v_scale, workspace)
    out = torch.empty_like(q)
    so = out.stride()
    lse = torch.empty((B, H, T), dtype=torch.float32, device=q.device)
    lib = load_library()
    if workspace is None:
        workspace = torch.empty(max(int(lib.flashmask_decode_workspace_bytes(B, H, heads, T, d)), 256), dtype=torch.uint8, device=q.device)
    _check(lib.flashmask_decode(cache, q.data_ptr(), lens_at, *at, columns, window, scale, out.data_ptr(), lse.data_ptr(),
                                _TYPE[q.dtype], H, T, (ctypes.c_int64 * 3)(*sq), (ctypes.c_int64 * 3)(*so[:3]), workspace.data_ptr(),
                                workspace.numel() * workspace.element_size(), _stream()), "flashmask_decode")
    return out, lse


def _pools(pools):
    """Addresses of page pools [pages, ...], their number, the bytes of a page, the pages."""
    if not pools:
        raise FlashMaskError("no pools")
    first = pools[0]
    shape, strides, dtype = first.shape, first.stride(), first.dtype
    entry = first.numel() // max(shape[0], 1)
    # a page is one run of memory: its axes in some order are dense
    dense = 1
    for stride, size in sorted(zip(strides[1:], shape[1:])):
        if size != 1:
            if stride != dense:
                raise FlashMaskError("a page of a pool must be one run of memory")
            dense *= size
    if len(shape) < 2 or (shape[0] > 1 and strides[0] != entry):
        raise FlashMaskError("a pool must be indexed [pages, ...], its pages one behind the other")
    for p in pools:
        if not p.is_cuda:
            raise FlashMaskError("the pools must live on the GPU")
        if p.shape != shape or p.stride() != strides or p.dtype is not dtype:
            raise FlashMaskError("the pools must have one shape, layout and type")
    return (ctypes.c_void_p * len(pools))(*[p.data_ptr() for p in pools]), len(pools), entry * first.element_size(), shape[0]


def flashmask_cache_fork(pools, table, lens, parents, new_pages, page: int):
    """Children that go on from sequences parents [children]: (table, lens) of the children.  Where new_pages[r] >= 0, child r's
    last page, if partly filled, is copied there in every pool (tensors [pages, ...] of `page` tokens to a page); -1: it goes on
    in its parent's."""
    where, n, page_bytes, num_pages = _pools(pools)
    if table.dim() != 2:
        raise FlashMaskError("table must be [sequences, columns]")
    B, columns = table.shape
    children = parents.shape[0] if parents.dim() == 1 else -1
    at = (_index(table, table.shape, "table"), _index(lens, (B,), "lens"), _index(parents, (children,), "parents"),
          _index(new_pages, (children,), "new_pages"))
    _same_device(table, lens, parents, new_pages, *pools)
    table_out = torch.empty((children, columns), dtype=torch.int32, device=table.device)
    lens_out = torch.empty(children, dtype=torch.int32, device=table.device)
    _check(load_library().flashmask_cache_fork(where, n, page_bytes, num_pages, *at, table_out.data_ptr(), lens_out.data_ptr(), B,
                                               columns, page, children, _stream()), "flashmask_cache_fork")
    return table_out, lens_out


def flashmask_cache_plan_bytes(num_pages: int) -> int:
    return int(load_library().flashmask_cache_plan_bytes(num_pages))


def _plan(lib, num_pages: int, device, workspace) -> torch.Tensor:
    if workspace is not None:
        return workspace
    return torch.empty(max(int(lib.flashmask_cache_plan_bytes(num_pages)), 256), dtype=torch.uint8, device=device)


def flashmask_cache_free_list(table, num_pages: int, workspace: torch.Tensor | None = None):
    """The pages that no entry of the table names, in ascending order with -1 behind them (int32 [num_pages]), and how many
    (int32 [1])."""
    at = _index(table, table.shape, "table")
    _same_device(table, workspace)
    lib = load_library()
    ws = _plan(lib, num_pages, table.device, workspace)
    if num_pages <= 0:
        raise FlashMaskError("num_pages must be positive")
    free = torch.empty(num_pages, dtype=torch.int32, device=table.device)
    count = torch.empty(1, dtype=torch.int32, device=table.device)
    _check(lib.flashmask_cache_free_list(at, table.numel(), num_pages, free.data_ptr(), count.data_ptr(), ws.data_ptr(),
                                         ws.numel() * ws.element_size(), _stream()), "flashmask_cache_free_list")
    return free, count


def flashmask_cache_compact(pools, table, workspace: torch.Tensor | None = None):
    """Move the pages that the table names to the front of every pool; (table, used) with the pages' new places and their
    number (int32 [1])."""
    where, n, page_bytes, num_pages = _pools(pools)
    at = _index(table, table.shape, "table")
    _same_device(table, workspace, *pools)
    lib = load_library()
    ws = _plan(lib, num_pages, table.device, workspace)
    table_out = torch.empty_like(table)
    used = torch.empty(1, dtype=torch.int32, device=table.device)
    _check(lib.flashmask_cache_compact(where, n, page_bytes, num_pages, at, table.numel(), table_out.data_ptr(), used.data_ptr(),
                                       ws.data_ptr(), ws.numel() * ws.element_size(), _stream()), "flashmask_cache_compact")
    return table_out, used
