"""Rotary positions, the paged key-value cache, attention of new tokens over it, and the weight of its keys (see include/flashmask.h for the contract).

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
_ONE, _TWO, _FOUR = struct.Struct("@3q"), struct.Struct("@6q"), struct.Struct("@12q")


# A call of few tokens takes the host longer than the GPU, so a call's checks are one expression, and what exactly is wrong is only
# looked for where it fails.
def _refuse(*wanted):
    """Raise what is wrong with tensors (t, name, types, shape, contiguous along how many of their last axes); something is."""
    device = torch._C._cuda_getDevice() if torch.cuda.is_available() else -1
    for t, name, types, shape, dense in wanted:
        if t is None:
            continue
        if not t.is_cuda:
            raise FlashMaskError(f"{name} must live on the GPU")
        if t.get_device() != device:
            raise FlashMaskError(f"the tensors must be on the current GPU, {device}: {name} is on {t.get_device()}")
        if t.dtype not in types:
            raise FlashMaskError(f"{name} must be {' or '.join(str(x) for x in types)}, got {t.dtype}")
        if t.dim() != len(shape) or any(want is not None and have != want for have, want in zip(t.shape, shape)):
            raise FlashMaskError(f"{name} must be [{', '.join('n' if x is None else str(x) for x in shape)}], got {list(t.shape)}")
        if 0 in t.shape:
            raise FlashMaskError(f"{name} is empty: {list(t.shape)}")
        if not (t.is_contiguous() if dense > 1 else t.stride(-1) == 1):
            raise FlashMaskError(f"{name} must be contiguous{'' if dense > 1 else ' along its last axis'}")
    raise FlashMaskError("the tensors do not go together")


# ctypes takes the lower 32 bits of a number that does not fit an int.
def _fits(*numbers) -> bool:
    return -1 << 31 <= min(numbers) and max(numbers) < 1 << 31


def _layout(layout):
    if layout not in (FM_ROPE_HALF, FM_ROPE_INTERLEAVED):
        raise FlashMaskError(f"layout must be FM_ROPE_HALF or FM_ROPE_INTERLEAVED, got {layout}")


def _rope(entry: str, q, k, freqs, positions, layout, amp):
    dtype, shape, sq, sk = q.dtype, q.shape, q.stride(), k.stride()
    type_id, device = _ROPE_TYPE.get(dtype), q.get_device()
    if not (type_id is not None and len(shape) == 4 and len(sk) == 4 and sq[3] == 1 and sk[3] == 1 and k.dtype is dtype
            and k.shape == (shape[0], k.shape[1], shape[2], shape[3]) and freqs.dtype is torch.float64 and freqs.dim() == 1
            and freqs.is_contiguous() and 0 <= device == k.get_device() == freqs.get_device() == torch._C._cuda_getDevice()
            and (positions is None or positions.dtype is torch.int32 and positions.shape == (shape[0], shape[2])
                 and positions.is_contiguous() and positions.get_device() == device)):
        like = (*shape, None, None, None, None)
        _refuse((q, "q", tuple(_ROPE_TYPE), (None,) * 4, 1), (k, "k", (dtype,), (like[0], None, like[2], like[3]), 1),
                (freqs, "freqs", (torch.float64,), (None,), 2), (positions, "positions", (torch.int32,), (like[0], like[2]), 2))
    _layout(layout)
    B, H, N, d = shape
    q_out, k_out = torch.empty_like(q), torch.empty_like(k)
    to_q, to_k = q_out.stride(), k_out.stride()
    strides = _FOUR.pack(sq[0], sq[1], sq[2], sk[0], sk[1], sk[2], to_q[0], to_q[1], to_q[2], to_k[0], to_k[1], to_k[2])
    _check(getattr(load_library(), entry)(q.data_ptr(), k.data_ptr(), q_out.data_ptr(), k_out.data_ptr(), freqs.data_ptr(),
                                          0 if positions is None else positions.data_ptr(), type_id, layout, amp, B, H, k.shape[1], N, d,
                                          2 * freqs.shape[0], strides, _stream()), entry)
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
    heads = shape[1] if len(shape) == 4 else None
    if not (type_id is not None and heads is not None and v_cache.shape == shape and v_cache.dtype is dtype and sk[3] == 1 and sv[3] == 1
            and len(entries) == 2 and table.dtype is torch.int32 and table.is_contiguous()
            and 0 <= device == k_cache.get_device() == v_cache.get_device() == table.get_device() == torch._C._cuda_getDevice()
            and (k_scale is None and v_scale is None or k_scale is not None and v_scale is not None
                 and k_scale.dtype is torch.float32 and v_scale.dtype is torch.float32 and k_scale.shape == (heads,) == v_scale.shape
                 and k_scale.is_contiguous() and v_scale.is_contiguous() and k_scale.get_device() == device == v_scale.get_device())):
        _refuse((k_cache, "k_cache", tuple(_CACHE_TYPE), (None,) * 4, 1), (v_cache, "v_cache", (dtype,), tuple(shape), 1),
                (table, "table", (torch.int32,), (None, None), 2), (k_scale, "k_scale", (torch.float32,), (heads,), 2),
                (v_scale, "v_scale", (torch.float32,), (heads,), 2))
    pages, _, page, d = shape
    sequences, columns = entries
    return (_CACHE.pack(k_cache.data_ptr(), v_cache.data_ptr(), sk[0], sk[1], sk[2], sv[0], sv[1], sv[2],
                        0 if k_scale is None else k_scale.data_ptr(), 0 if v_scale is None else v_scale.data_ptr(), table.data_ptr(),
                        type_id, heads, d, pages, page, sequences, columns), heads, d, sequences)


def flashmask_cache_append(k, v, k_cache, v_cache, table, seqs, positions, *, q=None, freqs=None, layout: int = FM_ROPE_HALF,
                           amp: float = 1.0, k_scale=None, v_scale=None):
    """Write new tokens' keys (rotated where freqs is given) and values [tokens, H_kv, d] to the cache: token n goes to position
    positions[n] of sequence seqs[n] (outside the table's sequences: padding).  Returns the queries q [tokens, H, d], rotated, or
    None."""
    dtype, shape, device, sk, sv = k.dtype, k.shape, k.get_device(), k.stride(), v.stride()
    type_id = _ROW_TYPE.get(dtype)
    cache, heads, d, _ = _cache(k_cache, v_cache, table, k_scale, v_scale, device)
    sq = (0, 0, 1) if q is None else q.stride()
    n = shape[0] if len(shape) == 3 else None
    if not (type_id is not None and shape == (n, heads, d) == v.shape and v.dtype is dtype and sk[2] == 1 and sv[2] == 1
            and seqs.dtype is torch.int32 and positions.dtype is torch.int32 and seqs.shape == (n,) == positions.shape
            and seqs.is_contiguous() and positions.is_contiguous() and device == v.get_device() == seqs.get_device() == positions.get_device()
            and (q is None or freqs is not None and len(sq) == 3 and sq[2] == 1 and q.dtype is dtype and q.shape == (n, q.shape[1], d)
                 and q.get_device() == device)
            and (freqs is None or freqs.dtype is torch.float64 and freqs.dim() == 1 and freqs.numel() > 0 and freqs.is_contiguous()
                 and freqs.get_device() == device)):
        if q is not None and freqs is None:
            raise FlashMaskError("q is only rotated: it needs freqs")
        _refuse((k, "k", tuple(_ROW_TYPE), (None, heads, d), 1), (v, "v", (dtype,), (n, heads, d), 1),
                (seqs, "seqs", (torch.int32,), (n,), 2), (positions, "positions", (torch.int32,), (n,), 2),
                (q, "q", (dtype,), (n, None, d), 1), (freqs, "freqs", (torch.float64,), (None,), 2))
    _layout(layout)
    H, q_at, out_at, q_out = 0, 0, 0, None
    if q is not None:
        H = q.shape[1]
        q_out = torch.empty(n, H, d, dtype=dtype, device=q.device)
        q_at, out_at = q.data_ptr(), q_out.data_ptr()
    if n == 0:
        return q_out
    strides = _FOUR.pack(0, sq[1], sq[0], 0, sk[1], sk[0], 0, sv[1], sv[0], 0, d, H * d)
    turned = 0 if freqs is None else freqs.data_ptr()
    _check(load_library().flashmask_cache_append(cache, q_at, k.data_ptr(), v.data_ptr(), out_at, seqs.data_ptr(), positions.data_ptr(),
                                                 turned, type_id, layout, amp, n, H, 2 * freqs.shape[0] if turned else 0, strides,
                                                 _stream()), "flashmask_cache_append")
    return q_out


def flashmask_decode_workspace_bytes(sequences: int, H: int, H_kv: int, T: int, d: int) -> int:
    return int(load_library().flashmask_decode_workspace_bytes(sequences, H, H_kv, T, d)) if _fits(sequences, H, H_kv, T, d) else 0


def flashmask_decode(q, k_cache, v_cache, table, lens, scale: float, *, bounds=None, window: int = 0, k_scale=None, v_scale=None,
                     workspace: torch.Tensor | None = None):
    """Attention of the last T (1 to 256) tokens of every sequence, q [sequences, H, T, d], over the cache, which holds lens[b] tokens of
    sequence b, the new ones among them.  bounds: (lts, lte, uts, ute), int32 [sequences, columns]; window: keys that a row sees,
    itself among them (0: all).  Returns out (laid out like q) and lse (fp32 [sequences, H, T])."""
    dtype, shape, device, sq = q.dtype, q.shape, q.get_device(), q.stride()
    type_id = _ROW_TYPE.get(dtype)
    cache, heads, d, B = _cache(k_cache, v_cache, table, k_scale, v_scale, device)
    if not (type_id is not None and len(shape) == 4 and shape[0] == B and shape[3] == d and sq[3] == 1 and lens.dtype is torch.int32
            and lens.shape == (B,) and lens.is_contiguous() and lens.get_device() == device
            and (workspace is None or workspace.get_device() == device and workspace.is_contiguous())):
        _refuse((q, "q", tuple(_ROW_TYPE), (B, None, None, d), 1), (lens, "lens", (torch.int32,), (B,), 2),
                *(() if workspace is None else ((workspace, "workspace", (workspace.dtype,), tuple(workspace.shape), 2),)))
    if not 0 <= window < 1 << 31:
        if window < 0:
            raise FlashMaskError(f"window must not be negative, got {window}")
        window = 0    # no table holds as many keys
    H, T = shape[1], shape[2]
    at, columns = (0, 0, 0, 0), 0
    if bounds is not None:
        if len(bounds) != 4:
            raise FlashMaskError("bounds must be (lts, lte, uts, ute), int32 [sequences, columns]")
        columns = bounds[0].shape[-1]
        for x in bounds:
            if not (x.dtype is torch.int32 and x.shape == (B, columns) and columns > 0 and x.is_contiguous() and x.get_device() == device):
                _refuse(*((y, n, (torch.int32,), (B, columns), 2) for y, n in zip(bounds, ("lts", "lte", "uts", "ute"))))
        at = [x.data_ptr() for x in bounds]
    out = torch.empty_like(q)
    so = out.stride()
    lse = torch.empty(B, H, T, dtype=torch.float32, device=q.device)
    lib = load_library()
    if workspace is None:
        workspace = torch.empty(max(int(lib.flashmask_decode_workspace_bytes(B, H, heads, T, d)), 256), dtype=torch.uint8, device=q.device)
    _check(lib.flashmask_decode(cache, q.data_ptr(), lens.data_ptr(), *at, columns, window, scale, out.data_ptr(), lse.data_ptr(), type_id, H, T,
                                _TWO.pack(sq[0], sq[1], sq[2], so[0], so[1], so[2]), workspace.data_ptr(),
                                workspace.numel() * workspace.element_size(), _stream()), "flashmask_decode")
    return out, lse


def _window(window):
    if not 0 <= window < 1 << 31:
        if window < 0:
            raise FlashMaskError(f"window must not be negative, got {window}")
        window = 0    # no table holds as many keys
    return window


def _bounds(bounds, B: int, device: int):
    """Addresses of (lts, lte, uts, ute) and their columns."""
    if bounds is None:
        return (0, 0, 0, 0), 0
    if len(bounds) != 4:
        raise FlashMaskError("bounds must be (lts, lte, uts, ute), int32 [sequences, columns]")
    columns = bounds[0].shape[-1] if bounds[0].dim() else 0
    for x in bounds:
        if not (x.dtype is torch.int32 and x.shape == (B, columns) and columns > 0 and x.is_contiguous() and x.get_device() == device):
            _refuse(*((y, n, (torch.int32,), (B, columns), 2) for y, n in zip(bounds, ("lts", "lte", "uts", "ute"))))
    return [x.data_ptr() for x in bounds], columns


def flashmask_decode_tree_workspace_bytes(sequences: int, H: int, H_kv: int, T: int, d: int) -> int:
    return int(load_library().flashmask_decode_tree_workspace_bytes(sequences, H, H_kv, T, d)) if _fits(sequences, H, H_kv, T, d) else 0


def flashmask_decode_tree(q, k_cache, v_cache, table, lens, parents, scale: float, *, bounds=None, window: int = 0, k_scale=None, v_scale=None,
                          workspace: torch.Tensor | None = None):
    """flashmask_decode where the last T tokens of a sequence are a tree of drafted ones: token t follows token parents[b, t] < t of them
    (int32 [sequences, T]; -1: the sequence ahead of them) and sees what is ahead of all of them, its ancestors and itself.  Its row, and its
    position, is lens[b] - T + the number of its ancestors."""
    dtype, shape, device, sq = q.dtype, q.shape, q.get_device(), q.stride()
    type_id = _ROW_TYPE.get(dtype)
    cache, heads, d, B = _cache(k_cache, v_cache, table, k_scale, v_scale, device)
    if not (type_id is not None and len(shape) == 4 and shape[0] == B and shape[3] == d and sq[3] == 1 and lens.dtype is torch.int32
            and lens.shape == (B,) and lens.is_contiguous() and parents.dtype is torch.int32 and parents.shape == (B, shape[2])
            and parents.is_contiguous() and device == lens.get_device() == parents.get_device()
            and (workspace is None or workspace.get_device() == device and workspace.is_contiguous())):
        _refuse((q, "q", tuple(_ROW_TYPE), (B, None, None, d), 1), (lens, "lens", (torch.int32,), (B,), 2),
                (parents, "parents", (torch.int32,), (B, shape[2] if len(shape) == 4 else None), 2),
                *(() if workspace is None else ((workspace, "workspace", (workspace.dtype,), tuple(workspace.shape), 2),)))
    window = _window(window)
    H, T = shape[1], shape[2]
    at, columns = _bounds(bounds, B, device)
    out = torch.empty_like(q)
    so = out.stride()
    lse = torch.empty(B, H, T, dtype=torch.float32, device=q.device)
    lib = load_library()
    if workspace is None:
        workspace = torch.empty(max(int(lib.flashmask_decode_tree_workspace_bytes(B, H, heads, T, d)), 256), dtype=torch.uint8, device=q.device)
    _check(lib.flashmask_decode_tree(cache, q.data_ptr(), lens.data_ptr(), parents.data_ptr(), *at, columns, window, scale, out.data_ptr(),
                                     lse.data_ptr(), type_id, H, T, _TWO.pack(sq[0], sq[1], sq[2], so[0], so[1], so[2]), workspace.data_ptr(),
                                     workspace.numel() * workspace.element_size(), _stream()), "flashmask_decode_tree")
    return out, lse


def flashmask_cache_accept(pools, table, lens, T: int, path):
    """Take over the accepted path of every sequence's tree of T drafted tokens, its last ones: token path[b, i] (int32 [sequences, n], ascending,
    -1 behind the last) moves to the i-th place behind the sequence ahead of them, in every pool (tensors [pages, heads, page, d] of one layout).
    Returns the new lengths."""
    if not pools:
        raise FlashMaskError("no pools")
    first = pools[0]
    shape, strides, dtype, device = first.shape, first.stride(), first.dtype, first.get_device()
    entries, ints = table.shape, torch.int32
    B = entries[0] if len(entries) == 2 else -1
    type_id = _CACHE_TYPE.get(dtype)
    if not (type_id is not None and len(shape) == 4 and strides[3] == 1 and table.dtype is ints and lens.dtype is ints
            and path.dtype is ints and lens.shape == (B,) and path.dim() == 2 and path.shape[0] == B and table.is_contiguous()
            and lens.is_contiguous() and path.is_contiguous()
            and 0 <= device == table.get_device() == lens.get_device() == path.get_device() == torch._C._cuda_getDevice()):
        _refuse((first, "pools", tuple(_CACHE_TYPE), (None,) * 4, 1), (table, "table", (ints,), (None, None), 2), (lens, "lens", (ints,), (B,), 2),
                (path, "path", (ints,), (B, None), 2))
    dense = first.is_contiguous()     # of contiguous tensors of one shape the strides need not be looked at
    for p in pools:
        if not (p.dtype is dtype and p.shape == shape and (p.is_contiguous() if dense else p.stride() == strides) and p.get_device() == device):
            raise FlashMaskError("the pools must have one shape, layout and type, on one GPU")
    if not _fits(T):
        raise FlashMaskError(f"T is out of range: {T}")
    at = [p.data_ptr() for p in pools]
    if len(set(at)) != len(at):
        raise FlashMaskError("a pool is named twice")
    pages, heads, page, d = shape
    lens_out = torch.empty_like(lens)
    _check(load_library().flashmask_cache_accept(struct.pack(f"@{len(at)}P", *at), len(at), _ONE.pack(*strides[:3]),
                                                 type_id, heads, d, pages, page, table.data_ptr(), lens.data_ptr(), path.data_ptr(),
                                                 lens_out.data_ptr(), B, entries[1], T, path.shape[1], _stream()), "flashmask_cache_accept")
    return lens_out


def flashmask_weights_workspace_bytes(B: int, H: int, H_kv: int, N: int, d: int, first_row: int = 0) -> int:
    return int(load_library().flashmask_weights_workspace_bytes(B, H, H_kv, N, d, first_row)) if _fits(B, H, H_kv, N, d, first_row) else 0


def flashmask_weights(q, k, lse, lts, lte, uts, ute, scale: float, *, first_row: int = 0, workspace: torch.Tensor | None = None):
    """The attention weight that each key of a prompt gets: fp32 [B,H_kv,N], sums of exp(scale q k - lse) over the rows from first_row on that see
    the key and the query heads of its K/V head.  q [B,H,N,d], k [B,H_kv,N,d] (bf16, any strides, d contiguous) and the bounds as for
    flashmask_fwd_ex, lse [B,H,N] from it."""
    shape, device, sq, sk = q.shape, q.get_device(), q.stride(), k.stride()
    bounds, ints, f32, half = (lts, lte, uts, ute), torch.int32, torch.float32, torch.bfloat16
    if not (len(shape) == 4 and q.dtype is half and k.dtype is half and sq[3] == 1 and len(sk) == 4 and sk[3] == 1
            and k.shape == (shape[0], k.shape[1], shape[2], shape[3]) and lse.dtype is f32 and lse.shape == shape[:3] and lse.is_contiguous()
            and 0 <= device == k.get_device() == lse.get_device() == torch._C._cuda_getDevice()
            and all(x.dtype is ints and x.shape == (shape[0], shape[2]) and x.is_contiguous() and x.get_device() == device for x in bounds)
            and (workspace is None or workspace.get_device() == device and workspace.is_contiguous())):
        like = (*shape, None, None, None, None)
        _refuse((q, "q", (half,), (None,) * 4, 1), (k, "k", (half,), (like[0], None, like[2], like[3]), 1), (lse, "lse", (f32,), like[:3], 2),
                *((x, n, (ints,), (like[0], like[2]), 2) for x, n in zip(bounds, ("lts", "lte", "uts", "ute"))),
                *(() if workspace is None else ((workspace, "workspace", (workspace.dtype,), tuple(workspace.shape), 2),)))
    B, H, N, d = shape
    heads = k.shape[1]
    if not _fits(first_row):
        raise FlashMaskError(f"first_row is out of range: {first_row}")
    lib = load_library()
    weights = torch.empty(B, heads, N, dtype=f32, device=q.device)
    if workspace is None:
        workspace = torch.empty(max(int(lib.flashmask_weights_workspace_bytes(B, H, heads, N, d, first_row)), 256), dtype=torch.uint8, device=q.device)
    _check(lib.flashmask_weights(q.data_ptr(), k.data_ptr(), lse.data_ptr(), *[x.data_ptr() for x in bounds], scale, weights.data_ptr(), B, H, heads,
                                 N, d, first_row, _TWO.pack(sq[0], sq[1], sq[2], sk[0], sk[1], sk[2]), workspace.data_ptr(),
                                 workspace.numel() * workspace.element_size(), _stream()), "flashmask_weights")
    return weights


def flashmask_cache_weights(q, k_cache, v_cache, table, lens, lse, scale: float, before=None, *, out=None, decay: float = 1.0, bounds=None,
                            window: int = 0, k_scale=None, v_scale=None):
    """Add the attention weight that the last T tokens of every sequence, q [sequences, H, T, d], give the cached keys: with lse, bounds and window of
    their flashmask_decode, out = decay * before + sums of exp(scale q k - lse) for the places of each sequence (those of its last T tokens:
    the sums alone); others stay as they are.  before, out: fp32 [sequences, H_kv, places]; without out it is before, and without both a
    new tensor of zeros for all places of the table.  Returns out."""
    dtype, shape, device, sq = q.dtype, q.shape, q.get_device(), q.stride()
    type_id, f32 = _ROW_TYPE.get(dtype), torch.float32
    cache, heads, d, B = _cache(k_cache, v_cache, table, k_scale, v_scale, device)
    if out is None:
        out = before if before is not None else torch.zeros(B, heads, table.shape[1] * k_cache.shape[2], dtype=f32, device=q.device)
    columns = out.shape[-1] if out.dim() else 0
    if not (type_id is not None and len(shape) == 4 and shape[0] == B and shape[3] == d and sq[3] == 1 and lens.dtype is torch.int32
            and lens.shape == (B,) and lens.is_contiguous() and lse.dtype is f32 and lse.shape == shape[:3] and lse.is_contiguous()
            and out.dtype is f32 and out.shape == (B, heads, columns) and out.is_contiguous()
            and device == lens.get_device() == lse.get_device() == out.get_device()
            and (before is None or before.dtype is f32 and before.shape == out.shape and before.is_contiguous() and before.get_device() == device)):
        _refuse((q, "q", tuple(_ROW_TYPE), (B, None, None, d), 1), (lens, "lens", (torch.int32,), (B,), 2), (lse, "lse", (f32,), tuple(shape[:3]), 2),
                (out, "out", (f32,), (B, heads, None), 2), (before, "before", (f32,), tuple(out.shape), 2))
    window = _window(window)
    at, bound_columns = _bounds(bounds, B, device)
    _check(load_library().flashmask_cache_weights(cache, q.data_ptr(), lens.data_ptr(), *at, bound_columns, window, scale, lse.data_ptr(),
                                                  0 if before is None else before.data_ptr(), decay, out.data_ptr(), columns, type_id, shape[1],
                                                  shape[2], _ONE.pack(sq[0], sq[1], sq[2]), _stream()), "flashmask_cache_weights")
    return out


def flashmask_cache_evict_workspace_bytes(sequences: int, weight_heads: int, weight_columns: int) -> int:
    return int(load_library().flashmask_cache_evict_workspace_bytes(sequences, weight_heads, weight_columns)) \
        if _fits(sequences, weight_heads, weight_columns) else 0


def flashmask_cache_evict(k_cache, v_cache, table, lens, weights, new_table, keep: int, *, first: int = 0, recent: int = 0, k_scale=None,
                          v_scale=None, workspace: torch.Tensor | None = None):
    """Sequences of more than `keep` tokens keep their `first` first, their `recent` last and the heaviest of the tokens between, in their order, in
    the pages new_table[b] (int32 [sequences, at least keep / page]).  weights fp32 [sequences, H_kv or 1, places]: a selection for each K/V head or
    one for all; equally heavy tokens: the first ones stay.  Returns table, lens, weights (of the tokens in their new places, 0 behind
    them) and the places that they come from (int32 [sequences, H_kv or 1, keep], -1 behind the last).  From then on places are not positions: the
    calls over the cache count rows, windows and bounds by place, and where each head keeps tokens of its own no bounds describe a sequence."""
    device, ints, f32 = k_cache.get_device(), torch.int32, torch.float32
    cache, heads, d, B = _cache(k_cache, v_cache, table, k_scale, v_scale, device)
    which, columns = weights.shape[1:] if weights.dim() == 3 else (heads, 0)
    if not (lens.dtype is ints and lens.shape == (B,) and lens.is_contiguous() and weights.dtype is f32 and weights.shape == (B, which, columns)
            and (which == heads or which == 1) and weights.is_contiguous() and new_table.dtype is ints and new_table.dim() == 2
            and new_table.shape[0] == B and new_table.is_contiguous() and device == lens.get_device() == weights.get_device() == new_table.get_device()
            and (workspace is None or workspace.get_device() == device and workspace.is_contiguous())):
        _refuse((lens, "lens", (ints,), (B,), 2), (weights, "weights", (f32,), (B, which if which in (heads, 1) else heads, None), 2),
                (new_table, "new_table", (ints,), (B, None), 2),
                *(() if workspace is None else ((workspace, "workspace", (workspace.dtype,), tuple(workspace.shape), 2),)))
    if not _fits(keep, first, recent):
        raise FlashMaskError(f"keep, first or recent is out of range: {keep}, {first}, {recent}")
    if not 0 < keep <= table.shape[1] * k_cache.shape[2]:
        raise FlashMaskError(f"keep must be positive and within the table's places, got {keep}")
    lib = load_library()
    if workspace is None:
        workspace = torch.empty(max(int(lib.flashmask_cache_evict_workspace_bytes(B, which, columns)), 256), dtype=torch.uint8, device=weights.device)
    table_out, lens_out, weights_out, kept = torch.empty_like(table), torch.empty_like(lens), torch.empty_like(weights), _ints(table, B, which, keep)
    _check(lib.flashmask_cache_evict(cache, lens.data_ptr(), weights.data_ptr(), which, columns, keep, first, recent, new_table.data_ptr(),
                                     new_table.shape[1], table_out.data_ptr(), lens_out.data_ptr(), weights_out.data_ptr(), kept.data_ptr(),
                                     workspace.data_ptr(), workspace.numel() * workspace.element_size(), _stream()), "flashmask_cache_evict")
    return table_out, lens_out, weights_out, kept


def _ints(like, *shape):
    return torch.empty(*shape, dtype=torch.int32, device=like.device)


def _pools(pools):
    """Addresses of page pools [pages, ...] as bytes, their number, the bytes of a page, the pages, the GPU."""
    if not pools:
        raise FlashMaskError("no pools")
    first = pools[0]
    shape, strides, dtype, device = first.shape, first.stride(), first.dtype, first.get_device()
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
    if device < 0 or device != torch._C._cuda_getDevice():
        _refuse((first, "pools", (dtype,), tuple(shape), 1))
    for p in pools:
        if not (p.dtype is dtype and p.shape == shape and p.stride() == strides and p.get_device() == device):
            raise FlashMaskError("the pools must have one shape, layout and type, on one GPU")
    return struct.pack(f"@{len(pools)}P", *[p.data_ptr() for p in pools]), len(pools), entry * first.element_size(), pages, device


def flashmask_cache_fork(pools, table, lens, parents, new_pages, page: int):
    """Children that go on from sequences parents [children]: (table, lens) of the children.  Where new_pages[r] >= 0, child r's
    last page, if partly filled, is copied there in every pool (tensors [pages, ...] of `page` tokens to a page); -1: it goes on
    in its parent's."""
    where, n, page_bytes, num_pages, device = _pools(pools)
    entries, whole, ints = table.shape, parents.shape, torch.int32
    if not (len(entries) == 2 and len(whole) == 1 and new_pages.shape == whole and lens.shape == (entries[0],) and table.dtype is ints
            and lens.dtype is ints and parents.dtype is ints and new_pages.dtype is ints and table.is_contiguous() and lens.is_contiguous()
            and parents.is_contiguous() and new_pages.is_contiguous()
            and device == table.get_device() == lens.get_device() == parents.get_device() == new_pages.get_device()):
        _refuse((table, "table", (ints,), (None, None), 2), (lens, "lens", (ints,), (entries[0],), 2), (parents, "parents", (ints,), (None,), 2),
                (new_pages, "new_pages", (ints,), tuple(whole), 2))
    if not _fits(page):
        raise FlashMaskError(f"page is out of range: {page}")
    B, columns = entries
    children = whole[0]
    table_out, lens_out = _ints(table, children, columns), _ints(table, children)
    _check(load_library().flashmask_cache_fork(where, n, page_bytes, num_pages, table.data_ptr(), lens.data_ptr(), parents.data_ptr(),
                                               new_pages.data_ptr(), table_out.data_ptr(), lens_out.data_ptr(), B, columns, page, children,
                                               _stream()), "flashmask_cache_fork")
    return table_out, lens_out


def flashmask_cache_plan_bytes(num_pages: int) -> int:
    return int(load_library().flashmask_cache_plan_bytes(num_pages)) if _fits(num_pages) else 0


def _plan(lib, num_pages: int, table, workspace, device: int) -> torch.Tensor:
    """The scratch of the two calls below, their table checked."""
    if not (table.dtype is torch.int32 and table.is_contiguous() and table.numel() > 0 and device == table.get_device()):
        _refuse((table, "table", (torch.int32,), tuple(table.shape), 2))
    if workspace is None:
        return torch.empty(max(int(lib.flashmask_cache_plan_bytes(num_pages)), 256), dtype=torch.uint8, device=table.device)
    if workspace.get_device() != device or not workspace.is_contiguous():
        _refuse((workspace, "workspace", (workspace.dtype,), tuple(workspace.shape), 2))
    return workspace


def flashmask_cache_free_list(table, num_pages: int, workspace: torch.Tensor | None = None):
    """The pages that no entry of the table names, in ascending order with -1 behind them (int32 [num_pages]), and how many
    (int32 [1])."""
    device = table.get_device()
    if device < 0 or device != torch._C._cuda_getDevice():
        _refuse((table, "table", (torch.int32,), tuple(table.shape), 2))
    if num_pages <= 0 or not _fits(num_pages):
        raise FlashMaskError(f"num_pages must be positive and fit 32 bits, got {num_pages}")
    lib = load_library()
    ws = _plan(lib, num_pages, table, workspace, device)
    free, count = _ints(table, num_pages), _ints(table, 1)
    _check(lib.flashmask_cache_free_list(table.data_ptr(), table.numel(), num_pages, free.data_ptr(), count.data_ptr(), ws.data_ptr(),
                                         ws.numel() * ws.element_size(), _stream()), "flashmask_cache_free_list")
    return free, count


def flashmask_cache_compact(pools, table, workspace: torch.Tensor | None = None):
    """Move the pages that the table names to the front of every pool; (table, used) with the pages' new places and their
    number (int32 [1])."""
    where, n, page_bytes, num_pages, device = _pools(pools)
    lib = load_library()
    ws = _plan(lib, num_pages, table, workspace, device)
    table_out, used = torch.empty_like(table), _ints(table, 1)
    _check(lib.flashmask_cache_compact(where, n, page_bytes, num_pages, table.data_ptr(), table.numel(), table_out.data_ptr(),
                                       used.data_ptr(), ws.data_ptr(), ws.numel() * ws.element_size(), _stream()),
           "flashmask_cache_compact")
    return table_out, used
