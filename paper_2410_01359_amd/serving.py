"""Rotary positions, the paged key-value cache and attention of new tokens over it (see include/flashmask.h for the contract).

Argument marshalling only, as in binding.py: every step runs in the HIP kernels, and nothing falls back.  A cache is a pair of
tensors indexed [pages, heads, tokens of a page, d] (any strides, d contiguous), a page table int32 [sequences, columns] with -1
where there is no page, and for 8-bit caches (torch.float8_e4m3fn) a scale for each head.
"""
from __future__ import annotations

import struct

import torch

from .binding import FlashMaskError, _check, _stream, load_library

FM_ROPE_HALF, FM_ROPE_INTERLEAVED = 0, 1

_ROPE_TYPE = {torch.bfloat16: 0, torch.float16: 1, torch.float32: 2}
_ROW_TYPE = {torch.bfloat16: 0, torch.float16: 1}
_CACHE_TYPE = {torch.bfloat16: 0, torch.float16: 1, torch.float8_e4m3fn: 3}
# flashmask_cache, and records of flashmask_strides one behind the other.  Packed by hand: a ctypes.Structure takes twice the time.
_CACHE = struct.Struct("@PP6qPPP7i")
_TWO, _FOUR = struct.Struct("@6q"), struct.Struct("@12q")


# Each check is one expression, and what exactly is wrong is only looked for where it fails: a call of one new token per
# sequence takes the host about as long as the GPU.
def _wrong(t, name: str, device: int, types=None, shape=None):
    """Raise what is wrong with a tensor (something is)."""
    if t.get_device() < 0:
        raise FlashMaskError(f"{name} must live on the GPU")
    if t.get_device() != device:
        raise FlashMaskError(f"the tensors must be on one GPU, the current one: {name} is on {t.get_device()}")
    if types is not None and t.dtype not in types:
        raise FlashMaskError(f"{name} must be {' or '.join(str(x) for x in types)}, got {t.dtype}")
    if shape is not None and tuple(t.shape) != tuple(shape):
        raise FlashMaskError(f"{name} must be {list(shape)}, got {list(t.shape)}")
    raise FlashMaskError(f"{name} must be contiguous (tensors of rows: along their rows)")


def _device(t, name: str) -> int:
    device = t.get_device()
    if device < 0 or device != torch._C._cuda_getDevice():
        _wrong(t, name, device if device < 0 else torch._C._cuda_getDevice())
    return device


def _index(t, shape, name: str, device: int) -> int:
    """Address of an int32 tensor of this shape."""
    if not (t.dtype is torch.int32 and t.shape == shape and t.is_contiguous() and t.get_device() == device):
        _wrong(t, name, device, (torch.int32,), shape)
    return t.data_ptr()


def _rows(t, shape, dtype, name: str, device: int):
    """Strides of a tensor of rows, the last of them 1."""
    strides = t.stride()
    if not (t.dtype is dtype and t.shape == shape and strides[-1] == 1 and t.get_device() == device):
        _wrong(t, name, device, (dtype,), shape)
    return strides


def _vector(t, n: int, dtype, name: str, device: int) -> int:
    """Address of a vector of n values (-1: of some); 0 for None."""
    if t is None:
        return 0
    if t.dim() != 1 or t.shape[0] != n and (n >= 0 or t.shape[0] == 0):
        raise FlashMaskError(f"{name} must be a vector of {n if n >= 0 else 'some'} values, got {list(t.shape)}")
    if not (t.dtype is dtype and t.is_contiguous() and t.get_device() == device):
        _wrong(t, name, device, (dtype,))
    return t.data_ptr()


def _dims(t, n: int, name: str):
    if t.dim() != n:
        raise FlashMaskError(f"{name} must have {n} dimensions, got {t.dim()}")
    return t.shape


def _rope(entry: str, q, k, freqs, positions, layout, amp):
    device, type_id, dtype = _device(q, "q"), _ROPE_TYPE.get(q.dtype), q.dtype
    if type_id is None:
        _wrong(q, "q", device, tuple(_ROPE_TYPE))
    B, H, N, d = shape = _dims(q, 4, "q")
    Hk = _dims(k, 4, "k")[1]
    sq, sk = _rows(q, shape, dtype, "q", device), _rows(k, (B, Hk, N, d), dtype, "k", device)
    at = 0 if positions is None else _index(positions, (B, N), "positions", device)
    frequencies = _vector(freqs, -1, torch.float64, "freqs", device)
    q_out, k_out = torch.empty_like(q), torch.empty_like(k)
    strides = _FOUR.pack(*sq[:3], *sk[:3], *q_out.stride()[:3], *k_out.stride()[:3])
    _check(getattr(load_library(), entry)(q.data_ptr(), k.data_ptr(), q_out.data_ptr(), k_out.data_ptr(), frequencies, at, type_id,
                                          layout, amp, B, H, Hk, N, d, 2 * freqs.shape[0], strides, _stream()), entry)
    return q_out, k_out


def flashmask_rope(q, k, freqs, positions=None, *, layout: int = FM_ROPE_HALF, amp: float = 1.0):
    """q [B,H,N,d] and k [B,H_kv,N,d] (bf16, fp16 or fp32; any strides, d contiguous) with their first 2 * len(freqs) elements
    turned by the angles positions * freqs (positions int32 [B,N], None: 0..N-1; freqs float64).  Laid out like q and k."""
    return _rope("flashmask_rope", q, k, freqs, positions, layout, amp)


def flashmask_rope_bwd(dq, dk, freqs, positions=None, *, layout: int = FM_ROPE_HALF, amp: float = 1.0):
    """The gradients of flashmask_rope's results to those of its q and k."""
    return _rope("flashmask_rope_bwd", dq, dk, freqs, positions, layout, amp)


def _cache(k_cache, v_cache, table, k_scale, v_scale, device: int):
    """flashmask_cache as bytes, and its heads, d and sequences."""
    dtype, shape, entries = k_cache.dtype, k_cache.shape, table.shape
    type_id, sk, sv = _CACHE_TYPE.get(dtype), k_cache.stride(), v_cache.stride()
    if not (type_id is not None and len(shape) == 4 and v_cache.shape == shape and v_cache.dtype is dtype and sk[3] == 1 and sv[3] == 1
            and len(entries) == 2 and table.dtype is torch.int32 and table.is_contiguous()
            and k_cache.get_device() == v_cache.get_device() == table.get_device() == device):
        _dims(k_cache, 4, "k_cache")
        for t, name, types, want in ((k_cache, "k_cache", tuple(_CACHE_TYPE), shape), (v_cache, "v_cache", (dtype,), shape),
                                     (table, "table", (torch.int32,), _dims(table, 2, "table"))):
            if t.dtype not in types or t.shape != want or t.get_device() != device or t.stride()[-1] != 1 or t is table and not t.is_contiguous():
                _wrong(t, name, device, types, want)
    pages, heads, page, d = shape
    sequences, columns = entries
    k_at = v_at = 0
    if k_scale is not None or v_scale is not None:
        k_at, v_at = (_vector(s, heads, torch.float32, n, device) for s, n in ((k_scale, "k_scale"), (v_scale, "v_scale")))
    return (_CACHE.pack(k_cache.data_ptr(), v_cache.data_ptr(), sk[0], sk[1], sk[2], sv[0], sv[1], sv[2], k_at, v_at, table.data_ptr(),
                        type_id, heads, d, pages, page, sequences, columns), heads, d, sequences)


def flashmask_cache_append(k, v, k_cache, v_cache, table, seqs, positions, *, q=None, freqs=None, layout: int = FM_ROPE_HALF,
                           amp: float = 1.0, k_scale=None, v_scale=None):
    """Write new tokens' keys (rotated where freqs is given) and values [tokens, H_kv, d] to the cache: token n goes to position
    positions[n] of sequence seqs[n] (outside the table's sequences: padding).  Returns the queries q [tokens, H, d], rotated, or
    None."""
    device, dtype = _device(k, "k"), k.dtype
    type_id = _ROW_TYPE.get(dtype)
    if type_id is None:
        _wrong(k, "k", device, tuple(_ROW_TYPE))
    cache, heads, d, _ = _cache(k_cache, v_cache, table, k_scale, v_scale, device)
    n = _dims(k, 3, "k")[0]
    sk, sv = _rows(k, (n, heads, d), dtype, "k", device), _rows(v, (n, heads, d), dtype, "v", device)
    seqs_at, positions_at = _index(seqs, (n,), "seqs", device), _index(positions, (n,), "positions", device)
    frequencies = _vector(freqs, -1, torch.float64, "freqs", device)
    H, q_at, out_at, q_out, sq = 0, 0, 0, None, (0, 0)
    if q is not None:
        if freqs is None:
            raise FlashMaskError("q is only rotated: it needs freqs")
        H = _dims(q, 3, "q")[1]
        sq = _rows(q, (n, H, d), dtype, "q", device)
        q_out = torch.empty(n, H, d, dtype=dtype, device=q.device)
        q_at, out_at = q.data_ptr(), q_out.data_ptr()
    if n == 0:
        return q_out
    strides = _FOUR.pack(0, sq[1], sq[0], 0, sk[1], sk[0], 0, sv[1], sv[0], 0, d, H * d)
    _check(load_library().flashmask_cache_append(cache, q_at, k.data_ptr(), v.data_ptr(), out_at, seqs_at, positions_at, frequencies,
                                                 type_id, layout, amp, n, H, 0 if freqs is None else 2 * freqs.shape[0], strides,
                                                 _stream()), "flashmask_cache_append")
    return q_out


def flashmask_decode_workspace_bytes(sequences: int, H: int, H_kv: int, T: int, d: int) -> int:
    return int(load_library().flashmask_decode_workspace_bytes(sequences, H, H_kv, T, d))


def flashmask_decode(q, k_cache, v_cache, table, lens, scale: float, *, bounds=None, window: int = 0, k_scale=None, v_scale=None,
                     workspace: torch.Tensor | None = None):
    """Attention of the last T (1 to 256) tokens of every sequence, q [sequences, H, T, d], over the cache, which holds lens[b] tokens of
    sequence b, the new ones among them.  bounds: (lts, lte, uts, ute), int32 [sequences, columns]; window: keys that a row sees,
    itself among them (0: all).  Returns out (laid out like q) and lse (fp32 [sequences, H, T])."""
    device, dtype = _device(q, "q"), q.dtype
    type_id = _ROW_TYPE.get(dtype)
    if type_id is None:
        _wrong(q, "q", device, tuple(_ROW_TYPE))
    cache, heads, d, sequences = _cache(k_cache, v_cache, table, k_scale, v_scale, device)
    B, H, T, _ = _dims(q, 4, "q")
    sq = _rows(q, (sequences, H, T, d), dtype, "q", device)
    lens_at = _index(lens, (B,), "lens", device)
    at, columns = (0, 0, 0, 0), 0
    if bounds is not None:
        if len(bounds) != 4 or bounds[0].numel() == 0:
            raise FlashMaskError("bounds must be (lts, lte, uts, ute), int32 [sequences, columns]")
        columns = bounds[0].shape[-1]
        at = [_index(x, (B, columns), n, device) for x, n in zip(bounds, ("lts", "lte", "uts", "ute"))]
    out = torch.empty_like(q)
    so = out.stride()
    lse = torch.empty(B, H, T, dtype=torch.float32, device=q.device)
    lib = load_library()
    if workspace is None:
        workspace = torch.empty(max(int(lib.flashmask_decode_workspace_bytes(B, H, heads, T, d)), 256), dtype=torch.uint8, device=q.device)
    elif workspace.get_device() != device or not workspace.is_contiguous():
        _wrong(workspace, "workspace", device)
    _check(lib.flashmask_decode(cache, q.data_ptr(), lens_at, *at, columns, window, scale, out.data_ptr(), lse.data_ptr(), type_id, H, T,
                                _TWO.pack(sq[0], sq[1], sq[2], so[0], so[1], so[2]), workspace.data_ptr(),
                                workspace.numel() * workspace.element_size(), _stream()), "flashmask_decode")
    return out, lse


def _ints(like, *shape):
    return torch.empty(*shape, dtype=torch.int32, device=like.device)


def _pools(pools):
    """Addresses of page pools [pages, ...] as bytes, their number, the bytes of a page, the pages, the GPU."""
    if not pools:
        raise FlashMaskError("no pools")
    first = pools[0]
    device = _device(first, "pools")
    shape, strides, dtype = first.shape, first.stride(), first.dtype
    pages = shape[0] if shape else 0
    entry = first.numel() // max(pages, 1)
    if not first.is_contiguous():
        # a page is one run of memory: its axes in some order are dense
        dense = 1
        for stride, size in sorted(zip(strides[1:], shape[1:])):
            if size != 1:
                if stride != dense:
                    raise FlashMaskError("a page of a pool must be one run of memory")
                dense *= size
    if len(shape) < 2 or pages > 1 and strides[0] != entry:
        raise FlashMaskError("a pool must be indexed [pages, ...], its pages one behind the other")
    for p in pools:
        if not (p.dtype is dtype and p.shape == shape and p.stride() == strides and p.get_device() == device):
            raise FlashMaskError("the pools must have one shape, layout and type, on one GPU")
    return struct.pack(f"@{len(pools)}P", *[p.data_ptr() for p in pools]), len(pools), entry * first.element_size(), pages, device


def flashmask_cache_fork(pools, table, lens, parents, new_pages, page: int):
    """Children that go on from sequences parents [children]: (table, lens) of the children.  Where new_pages[r] >= 0, child r's
    last page, if partly filled, is copied there in every pool (tensors [pages, ...] of `page` tokens to a page); -1: it goes on
    in its parent's."""
    where, n, page_bytes, num_pages, device = _pools(pools)
    B, columns = entries = _dims(table, 2, "table")
    children = _dims(parents, 1, "parents")[0]
    at = (_index(table, entries, "table", device), _index(lens, (B,), "lens", device),
          _index(parents, (children,), "parents", device), _index(new_pages, (children,), "new_pages", device))
    table_out, lens_out = _ints(table, children, columns), _ints(table, children)
    _check(load_library().flashmask_cache_fork(where, n, page_bytes, num_pages, *at, table_out.data_ptr(), lens_out.data_ptr(), B,
                                               columns, page, children, _stream()), "flashmask_cache_fork")
    return table_out, lens_out


def flashmask_cache_plan_bytes(num_pages: int) -> int:
    return int(load_library().flashmask_cache_plan_bytes(num_pages))


def _plan(lib, num_pages: int, table, workspace, device: int) -> torch.Tensor:
    if workspace is None:
        return torch.empty(max(int(lib.flashmask_cache_plan_bytes(num_pages)), 256), dtype=torch.uint8, device=table.device)
    if workspace.get_device() != device or not workspace.is_contiguous():
        _wrong(workspace, "workspace", device)
    return workspace


def flashmask_cache_free_list(table, num_pages: int, workspace: torch.Tensor | None = None):
    """The pages that no entry of the table names, in ascending order with -1 behind them (int32 [num_pages]), and how many
    (int32 [1])."""
    device = _device(table, "table")
    at = _index(table, table.shape, "table", device)
    if num_pages <= 0:
        raise FlashMaskError("num_pages must be positive")
    lib = load_library()
    ws = _plan(lib, num_pages, table, workspace, device)
    free, count = _ints(table, num_pages), _ints(table, 1)
    _check(lib.flashmask_cache_free_list(at, table.numel(), num_pages, free.data_ptr(), count.data_ptr(), ws.data_ptr(),
                                         ws.numel() * ws.element_size(), _stream()), "flashmask_cache_free_list")
    return free, count


def flashmask_cache_compact(pools, table, workspace: torch.Tensor | None = None):
    """Move the pages that the table names to the front of every pool; (table, used) with the pages' new places and their
    number (int32 [1])."""
    where, n, page_bytes, num_pages, device = _pools(pools)
    at = _index(table, table.shape, "table", device)
    lib = load_library()
    ws = _plan(lib, num_pages, table, workspace, device)
    table_out, used = torch.empty_like(table), _ints(table, 1)
    _check(lib.flashmask_cache_compact(where, n, page_bytes, num_pages, at, table.numel(), table_out.data_ptr(), used.data_ptr(),
                                       ws.data_ptr(), ws.numel() * ws.element_size(), _stream()), "flashmask_cache_compact")
    return table_out, used
