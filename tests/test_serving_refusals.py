"""No GPU: the entry points around the attention call refuse unusable arguments before anything touches a device.  (The C entries
are given addresses that are never followed; every call here is refused.)"""
import ctypes
import struct

import pytest
import torch

import paper_2410_01359_amd as fm

OK, NULL, SHAPE, ALIGN, WORKSPACE, ARG = 0, -1, -2, -3, -4, -6
P = 1 << 20   # an aligned address
BF16, F16, F32, E4M3 = 0, 1, 2, 3


def _cache(k=P, v=P, sk=(8 * 64 * 128, 64 * 128, 128), sv=(8 * 64 * 128, 64 * 128, 128), k_scale=0, v_scale=0, table=P, type=BF16,
           heads=8, d=128, num_pages=10, page=64, sequences=3, columns=4):
    return struct.pack("@PP6qPPP7i", k, v, *sk, *sv, k_scale, v_scale, table, type, heads, d, num_pages, page, sequences, columns)


def _longs(*x):
    return (ctypes.c_int64 * len(x))(*x)


def _rope(entry="flashmask_rope", q=P, k=P, qo=P, ko=P, freqs=P, type=BF16, layout=0, amp=1.0, B=2, H=4, Hk=2, N=100, d=128, rot=128,
          strides=(51200, 12800, 128) * 4):
    return getattr(fm.load_library(), entry)(q, k, qo, ko, freqs, None, type, layout, amp, B, H, Hk, N, d, rot,
                                             None if strides is None else _longs(*strides), None)


@pytest.mark.parametrize("entry", ["flashmask_rope", "flashmask_rope_bwd"])
@pytest.mark.parametrize("wrong,code", [
    ({"q": None}, NULL), ({"k": None}, NULL), ({"qo": None}, NULL), ({"ko": None}, NULL), ({"freqs": None}, NULL), ({"strides": None}, NULL),
    ({"type": E4M3}, ARG), ({"type": 9}, ARG), ({"layout": 2}, ARG), ({"amp": float("nan")}, ARG), ({"amp": float("inf")}, ARG),
    ({"B": 0}, SHAPE), ({"H": 0}, SHAPE), ({"Hk": -1}, SHAPE), ({"N": 0}, SHAPE), ({"d": 96}, SHAPE), ({"rot": 0}, SHAPE),
    ({"rot": 24}, SHAPE), ({"rot": 144}, SHAPE), ({"N": 1 << 30}, SHAPE), ({"q": P + 8}, ALIGN), ({"ko": P + 2}, ALIGN),
    ({"strides": (51200, 12800, 132) * 4}, ALIGN), ({"strides": (51200, 12800, 64) * 4}, SHAPE),
    ({"strides": (0, 12800, 128) * 4}, SHAPE), ({"strides": (51200, 0, 128) * 4}, SHAPE), ({"strides": (51200, 12800, 1 << 24) * 4}, SHAPE)])
def test_rope(entry, wrong, code):
    assert _rope(entry, **wrong) == code


def _append(cache=None, q=P, k=P, v=P, qo=P, seqs=P, positions=P, freqs=P, type=BF16, layout=0, amp=1.0, tokens=5, H=16, rot=64,
            strides=(0, 128, 4096) * 4):
    return fm.load_library().flashmask_cache_append(_cache() if cache is None else cache, q, k, v, qo, seqs, positions, freqs, type, layout,
                                                    amp, tokens, H, rot, _longs(*strides), None)


def _decode(cache=None, q=P, lens=P, bounds=(None,) * 4, columns=0, window=0, scale=0.1, out=P, lse=P, type=BF16, H=16, T=2,
            sq=(4096, 256, 128), so=(4096, 256, 128), workspace=P, nbytes=1 << 40):
    return fm.load_library().flashmask_decode(_cache() if cache is None else cache, q, lens, *bounds, columns, window, scale, out, lse, type,
                                              H, T, _longs(*sq, *so), workspace, nbytes, None)


@pytest.mark.parametrize("call", [_append, _decode])
@pytest.mark.parametrize("wrong,code", [
    ({"k": 0}, NULL), ({"v": 0}, NULL), ({"table": 0}, NULL), ({"k_scale": P}, NULL), ({"v_scale": P}, NULL), ({"type": E4M3}, NULL),
    ({"type": E4M3, "k_scale": P}, NULL), ({"type": F32}, ARG), ({"type": F16}, ARG), ({"heads": 0}, SHAPE), ({"d": 32}, SHAPE),
    ({"num_pages": 0}, SHAPE), ({"page": 0}, SHAPE), ({"page": 24}, SHAPE), ({"page": 1 << 21}, SHAPE), ({"sequences": 0}, SHAPE),
    ({"columns": 0}, SHAPE), ({"columns": 1 << 25}, SHAPE), ({"k": P + 4}, ALIGN), ({"v": P + 8}, ALIGN),
    ({"sk": (65536, 8192, 132)}, ALIGN), ({"sv": (65536, 8192, 64)}, SHAPE), ({"sk": (65536, 0, 128)}, SHAPE), ({"sv": (65540, 8192, 128)}, ALIGN),
    ({"sk": (-65536, 8192, 128)}, SHAPE), ({"sk": (65536, 8192, 1 << 24)}, SHAPE)])
def test_unusable_caches(call, wrong, code):
    assert call(cache=_cache(**wrong)) == code
    assert call(cache=0) == NULL


@pytest.mark.parametrize("wrong,code", [
    ({"k": None}, NULL), ({"v": None}, NULL), ({"seqs": None}, NULL), ({"positions": None}, NULL), ({"qo": None}, NULL), ({"freqs": None}, NULL),
    ({"type": F32}, ARG), ({"type": F16}, ARG), ({"layout": -1}, ARG), ({"amp": float("nan")}, ARG), ({"tokens": 0}, SHAPE), ({"H": 0}, SHAPE),
    ({"rot": 8}, SHAPE), ({"rot": 256}, SHAPE), ({"q": P + 2}, ALIGN), ({"strides": (0, 128, 4100) * 4}, ALIGN), ({"strides": (0, 128, 64) * 4}, SHAPE)])
def test_append(wrong, code):
    assert _append(**wrong) == code


@pytest.mark.parametrize("wrong,code", [
    ({"q": None}, NULL), ({"lens": None}, NULL), ({"out": None}, NULL), ({"lse": None}, NULL), ({"bounds": (P, P, P, None)}, NULL),
    ({"bounds": (None, None, P, None)}, NULL), ({"type": F32}, ARG), ({"scale": 0.0}, ARG), ({"scale": float("nan")}, ARG),
    ({"scale": float("inf")}, ARG), ({"window": -1}, ARG), ({"H": 12}, SHAPE), ({"H": 0}, SHAPE), ({"T": 0}, SHAPE), ({"T": 257}, SHAPE),
    ({"bounds": (P,) * 4}, SHAPE), ({"sq": (4096, 256, 120)}, SHAPE), ({"so": (4100, 256, 128)}, ALIGN), ({"q": P + 8}, ALIGN),
    ({"workspace": None}, WORKSPACE), ({"workspace": P + 16}, WORKSPACE), ({"nbytes": 100}, WORKSPACE)])
def test_decode(wrong, code):
    assert _decode(**wrong) == code


def test_tables_beyond_32_bits_of_keys_are_refused():
    assert _decode(cache=_cache(sequences=100, columns=1 << 20, page=256)) == SHAPE
    assert _decode(cache=_cache(sequences=65535, heads=1024, sk=(1 << 23, 8192, 128), sv=(1 << 23, 8192, 128)), H=1024, T=1,
                   sq=(1 << 17, 128, 128), so=(1 << 17, 128, 128)) == SHAPE


def test_decode_workspace_bytes():
    size = fm.flashmask_decode_workspace_bytes
    for bad in ((0, 8, 8, 1, 128), (1, 0, 1, 1, 128), (1, 8, 3, 1, 128), (1, 8, 0, 1, 128), (1, 8, 8, 0, 128), (1, 8, 8, 1, 96)):
        assert size(*bad) == 0
    for B in (1, 64, 1000):
        for H, Hk, T, d in ((8, 8, 1, 128), (32, 4, 4, 64), (128, 16, 8, 128), (8, 1, 8, 64)):
            assert 0 < size(B, H, Hk, T, d) <= 64 << 20


def _pools(*p):
    return (ctypes.c_void_p * max(len(p), 1))(*p)


@pytest.mark.parametrize("wrong,code", [
    ({"pools": None}, NULL), ({"pools": _pools(P, 0)}, NULL), ({"pools": _pools(P, P + 8)}, ALIGN), ({"n": -1}, SHAPE), ({"nbytes": 0}, SHAPE),
    ({"nbytes": 40}, SHAPE), ({"num_pages": 0}, SHAPE), ({"table": None}, NULL), ({"lens": None}, NULL), ({"parents": None}, NULL),
    ({"new": None}, NULL), ({"table_out": None}, NULL), ({"lens_out": None}, NULL), ({"B": 0}, SHAPE), ({"columns": 0}, SHAPE),
    ({"page": 0}, SHAPE), ({"children": 0}, SHAPE), ({"children": 70000}, SHAPE)])
def test_fork(wrong, code):
    a = {"pools": _pools(P, P), "n": 2, "nbytes": 4096, "num_pages": 9, "table": P, "lens": P, "parents": P, "new": P, "table_out": P,
         "lens_out": P, "B": 2, "columns": 3, "page": 16, "children": 4} | wrong
    assert fm.load_library().flashmask_cache_fork(*a.values(), None) == code


def test_free_list_and_compact():
    lib = fm.load_library()
    need = fm.flashmask_cache_plan_bytes(100)
    assert need > 0 and fm.flashmask_cache_plan_bytes(0) == 0

    def free(table=P, entries=7, pages=100, out=P, count=P, ws=P, nbytes=need):
        return lib.flashmask_cache_free_list(table, entries, pages, out, count, ws, nbytes, None)

    def compact(pools=_pools(P), n=1, page_bytes=4096, pages=100, table=P, entries=7, out=P, used=P, ws=P, nbytes=need):
        return lib.flashmask_cache_compact(pools, n, page_bytes, pages, table, entries, out, used, ws, nbytes, None)

    for call in (free, compact):
        assert call(table=None) == NULL and call(out=None) == NULL
        assert call(entries=0) == SHAPE and call(pages=0) == SHAPE
        assert call(ws=None) == WORKSPACE and call(ws=P + 128) == WORKSPACE and call(nbytes=need - 1) == WORKSPACE
    assert free(count=None) == NULL and compact(used=None) == NULL
    assert compact(pools=None) == NULL and compact(page_bytes=24) == SHAPE and compact(pools=_pools(P + 4)) == ALIGN


def test_tensors_on_the_host_are_refused():
    bf = lambda *s: torch.zeros(s, dtype=torch.bfloat16)   # noqa: E731
    ints = lambda *s: torch.zeros(s, dtype=torch.int32)    # noqa: E731
    cache = (bf(3, 2, 16, 64), bf(3, 2, 16, 64), ints(1, 2))
    freqs = torch.ones(8, dtype=torch.float64)
    for call in (lambda: fm.flashmask_rope(bf(1, 2, 4, 64), bf(1, 2, 4, 64), freqs),
                 lambda: fm.flashmask_rope_bwd(bf(1, 2, 4, 64), bf(1, 2, 4, 64), freqs),
                 lambda: fm.flashmask_cache_append(bf(4, 2, 64), bf(4, 2, 64), *cache, ints(4), ints(4)),
                 lambda: fm.flashmask_decode(bf(1, 2, 1, 64), *cache, ints(1), 1.0),
                 lambda: fm.flashmask_cache_fork([cache[0]], cache[2], ints(1), ints(1), ints(1), 16),
                 lambda: fm.flashmask_cache_fork([], cache[2], ints(1), ints(1), ints(1), 16),
                 lambda: fm.flashmask_cache_free_list(cache[2], 3),
                 lambda: fm.flashmask_cache_compact([cache[0]], cache[2])):
        with pytest.raises(fm.FlashMaskError):
            call()
