"""The entry points for weights of keys, eviction and trees of drafted tokens refuse unusable arguments before anything touches a device (the C
entries are given addresses that are never followed; every call of them here is refused), and so does the binding."""
import ctypes
import struct

import pytest
import torch

import paper_2410_01359_amd as fm

NULL, SHAPE, ALIGN, WORKSPACE, ARG = -1, -2, -3, -4, -6
P = 1 << 20   # an aligned address
BF16, F16, F32, E4M3 = 0, 1, 2, 3
BEYOND = 1 << 32


def _cache(k=P, v=P, sk=(8 * 64 * 128, 64 * 128, 128), sv=(8 * 64 * 128, 64 * 128, 128), k_scale=0, v_scale=0, table=P, type=BF16,
           heads=8, d=128, num_pages=10, page=64, sequences=3, columns=4):
    return struct.pack("@PP6qPPP7i", k, v, *sk, *sv, k_scale, v_scale, table, type, heads, d, num_pages, page, sequences, columns)


def _longs(*x):
    return (ctypes.c_int64 * len(x))(*x)


def _pools(*p):
    return (ctypes.c_void_p * max(len(p), 1))(*p)


def _tree(cache=None, q=P, lens=P, parents=P, bounds=(None,) * 4, columns=0, window=0, scale=0.1, out=P, lse=P, type=BF16, H=16, T=5,
          sq=(10240, 640, 128), so=(10240, 640, 128), workspace=P, nbytes=1 << 40):
    return fm.load_library().flashmask_decode_tree(_cache() if cache is None else cache, q, lens, parents, *bounds, columns, window, scale, out, lse,
                                                   type, H, T, _longs(*sq, *so), workspace, nbytes, None)


def _cache_weights(cache=None, q=P, lens=P, bounds=(None,) * 4, columns=0, window=0, scale=0.1, lse=P, before=P, decay=1.0, weights=P,
                   places=256, type=BF16, H=16, T=5, sq=(10240, 640, 128)):
    return fm.load_library().flashmask_cache_weights(_cache() if cache is None else cache, q, lens, *bounds, columns, window, scale, lse, before,
                                                     decay, weights, places, type, H, T, None if sq is None else _longs(*sq), None)


def _evict(cache=None, lens=P, weights=P, heads=8, places=256, keep=100, first=2, recent=10, new_table=P, new_columns=2, table_out=P, lens_out=P,
           weights_out=P, kept=P, workspace=P, nbytes=1 << 40):
    return fm.load_library().flashmask_cache_evict(_cache() if cache is None else cache, lens, weights, heads, places, keep, first, recent, new_table,
                                                   new_columns, table_out, lens_out, weights_out, kept, workspace, nbytes, None)


@pytest.mark.parametrize("call", [_tree, _cache_weights, _evict])
@pytest.mark.parametrize("wrong,code", [
    ({"k": 0}, NULL), ({"v": 0}, NULL), ({"table": 0}, NULL), ({"k_scale": P}, NULL), ({"type": E4M3}, NULL), ({"type": E4M3, "k_scale": P}, NULL),
    ({"type": F32}, ARG), ({"heads": 0}, SHAPE), ({"d": 32}, SHAPE), ({"num_pages": 0}, SHAPE), ({"page": 24}, SHAPE), ({"page": 1 << 21}, SHAPE),
    ({"sequences": 0}, SHAPE), ({"columns": 0}, SHAPE), ({"columns": 1 << 25}, SHAPE), ({"k": P + 4}, ALIGN), ({"sk": (65536, 8192, 132)}, ALIGN),
    ({"sv": (65536, 8192, 64)}, SHAPE), ({"sk": (-65536, 8192, 128)}, SHAPE)])
def test_unusable_caches(call, wrong, code):
    assert call(cache=_cache(**wrong)) == code
    assert call(cache=0) == NULL


@pytest.mark.parametrize("wrong,code", [
    ({"q": None}, NULL), ({"lens": None}, NULL), ({"parents": None}, NULL), ({"out": None}, NULL), ({"lse": None}, NULL),
    ({"bounds": (P, P, P, None)}, NULL), ({"type": F32}, ARG), ({"type": F16}, ARG), ({"scale": 0.0}, ARG), ({"scale": float("inf")}, ARG),
    ({"window": -1}, ARG), ({"H": 12}, SHAPE), ({"T": 0}, SHAPE), ({"T": 257}, SHAPE), ({"bounds": (P,) * 4}, SHAPE), ({"sq": (10240, 640, 120)}, SHAPE),
    ({"so": (10244, 640, 128)}, ALIGN), ({"q": P + 8}, ALIGN), ({"workspace": None}, WORKSPACE), ({"workspace": P + 16}, WORKSPACE), ({"nbytes": 9}, WORKSPACE)])
def test_tree(wrong, code):
    assert _tree(**wrong) == code


@pytest.mark.parametrize("wrong,code", [
    ({"q": None}, NULL), ({"lens": None}, NULL), ({"lse": None}, NULL), ({"weights": None}, NULL), ({"sq": None}, NULL), ({"bounds": (None, P, P, P)}, NULL),
    ({"type": F32}, ARG), ({"type": F16}, ARG), ({"scale": -1.0}, ARG), ({"scale": float("nan")}, ARG), ({"window": -1}, ARG), ({"decay": -0.5}, ARG),
    ({"decay": float("nan")}, ARG), ({"decay": float("inf")}, ARG), ({"H": 12}, SHAPE), ({"H": 0}, SHAPE), ({"T": 0}, SHAPE), ({"T": 257}, SHAPE),
    ({"places": 0}, SHAPE), ({"places": (1 << 30) + 1}, SHAPE), ({"bounds": (P,) * 4}, SHAPE), ({"sq": (10240, 640, 120)}, SHAPE),
    ({"sq": (10244, 640, 128)}, ALIGN), ({"q": P + 8}, ALIGN)])
def test_cache_weights(wrong, code):
    assert _cache_weights(**wrong) == code


def test_cache_weights_of_too_many_chunks():
    assert _cache_weights(cache=_cache(sequences=60000, columns=1 << 20, page=1024), places=1 << 30) == SHAPE


@pytest.mark.parametrize("wrong,code", [
    ({"lens": None}, NULL), ({"weights": None}, NULL), ({"new_table": None}, NULL), ({"table_out": None}, NULL), ({"lens_out": None}, NULL),
    ({"weights_out": None}, NULL), ({"kept": None}, NULL), ({"heads": 2}, SHAPE), ({"heads": 0}, SHAPE), ({"places": 0}, SHAPE), ({"keep": 0}, SHAPE),
    ({"keep": -1}, SHAPE), ({"first": -1}, SHAPE), ({"recent": -1}, SHAPE), ({"first": 95}, SHAPE), ({"recent": 2 ** 31 - 1}, SHAPE),
    ({"new_columns": 1}, SHAPE), ({"new_columns": 0}, SHAPE), ({"keep": 257, "new_columns": 5}, SHAPE), ({"workspace": None}, WORKSPACE),
    ({"workspace": P + 16}, WORKSPACE), ({"nbytes": 0}, WORKSPACE)])
def test_evict(wrong, code):
    assert _evict(**wrong) == code


@pytest.mark.parametrize("wrong,code", [
    ({"pools": None}, NULL), ({"pools": _pools(P, 0)}, NULL), ({"pools": _pools(P, P + 8)}, ALIGN), ({"n": 0}, SHAPE), ({"strides": None}, NULL),
    ({"type": F32}, ARG), ({"heads": 0}, SHAPE), ({"d": 96}, SHAPE), ({"num_pages": 0}, SHAPE), ({"page": 24}, SHAPE), ({"table": None}, NULL),
    ({"lens": None}, NULL), ({"path": None}, NULL), ({"lens_out": None}, NULL), ({"B": 0}, SHAPE), ({"B": 65536}, SHAPE), ({"columns": 0}, SHAPE),
    ({"columns": 1 << 28}, SHAPE), ({"T": 0}, SHAPE), ({"T": 257}, SHAPE), ({"P": 0}, SHAPE), ({"P": 8}, SHAPE),
    ({"strides": _longs(65536, 8192, 132)}, ALIGN), ({"strides": _longs(65536, 8192, 64)}, SHAPE)])
def test_accept(wrong, code):
    a = {"pools": _pools(P, P), "n": 2, "strides": _longs(65536, 8192, 128), "type": BF16, "heads": 8, "d": 128, "num_pages": 9, "page": 64, "table": P,
         "lens": P, "path": P, "lens_out": P, "B": 2, "columns": 3, "T": 7, "P": 4} | wrong
    assert fm.load_library().flashmask_cache_accept(*a.values(), None) == code


def _weights(q=P, k=P, lse=P, lts=P, lte=P, uts=P, ute=P, scale=0.1, weights=P, B=2, H=4, Hk=2, N=100, d=128, first_row=0,
             strides=(51200, 12800, 128) * 2, ws=P, nbytes=1 << 40):
    return fm.load_library().flashmask_weights(q, k, lse, lts, lte, uts, ute, scale, weights, B, H, Hk, N, d, first_row,
                                               None if strides is None else _longs(*strides), ws, nbytes, None)


@pytest.mark.parametrize("wrong,code", [
    *(({n: None}, NULL) for n in ("q", "k", "lse", "lts", "lte", "uts", "ute", "weights", "strides")), ({"scale": 0.0}, ARG),
    ({"scale": float("nan")}, ARG), ({"B": 0}, SHAPE), ({"H": 3}, SHAPE), ({"H": 0}, SHAPE), ({"Hk": 0}, SHAPE), ({"N": 0}, SHAPE), ({"d": 96}, SHAPE),
    ({"first_row": -1}, SHAPE), ({"first_row": 100}, SHAPE), ({"N": (1 << 30) + 1}, SHAPE), ({"B": 1 << 24}, SHAPE), ({"q": P + 8}, ALIGN), ({"k": P + 2}, ALIGN),
    ({"strides": (51200, 12800, 132) * 2}, ALIGN), ({"strides": (51200, 12800, 64) * 2}, SHAPE), ({"ws": None}, WORKSPACE), ({"ws": P + 128}, WORKSPACE),
    ({"nbytes": 0}, WORKSPACE)])
def test_weights(wrong, code):
    assert _weights(**wrong) == code


def test_sizes_of_scratch():
    of_weights, of_evict = fm.flashmask_weights_workspace_bytes, fm.flashmask_cache_evict_workspace_bytes
    assert of_weights(1, 32, 8, 1000, 128) > 0 and of_weights(1, 32, 8, 1000, 128, 999) > 0 and of_evict(2, 8, 1000) > 0
    for bad in ((0, 8, 8, 10, 64), (1, 8, 3, 10, 64), (1, 8, 8, 0, 64), (1, 8, 8, 10, 96), (1, 8, 8, 10, 64, 10), (1, 8, 8, 10, 64, -1)):
        assert of_weights(*bad) == 0
    for bad in ((0, 8, 10), (1, 0, 10), (1, 8, 0), (70000, 8, 10)):
        assert of_evict(*bad) == 0
    of_tree = fm.flashmask_decode_tree_workspace_bytes
    assert of_tree(2, 8, 2, 5, 64) > 0 and 0 < of_tree(2, 32, 8, 256, 128) <= 1 << 28
    for bad in ((0, 8, 8, 1, 128), (1, 0, 1, 1, 128), (1, 8, 3, 1, 128), (1, 8, 0, 1, 128), (1, 8, 8, 0, 128), (1, 8, 8, 257, 128), (1, 8, 8, 1, 96)):
        assert of_tree(*bad) == 0
    for at in range(5):
        shape = [2, 8, 2, 5, 64]
        shape[at] += BEYOND
        assert of_tree(*shape) == 0
    for at in range(6):
        shape = [1, 8, 2, 100, 64, 5]
        shape[at] += BEYOND
        assert of_weights(*shape) == 0
    for at in range(3):
        shape = [1, 8, 100]
        shape[at] -= BEYOND
        assert of_evict(*shape) == 0


def _tensors(device):
    bf = lambda *s: torch.zeros(s, dtype=torch.bfloat16, device=device)   # noqa: E731
    ints = lambda *s: torch.zeros(s, dtype=torch.int32, device=device)    # noqa: E731
    floats = lambda *s: torch.zeros(s, device=device)                     # noqa: E731
    pool = {"k_cache": bf(6, 2, 16, 64), "v_cache": bf(6, 2, 16, 64), "table": ints(1, 2), "lens": ints(1)}
    bounds = {n: ints(1, 20) for n in ("lts", "lte", "uts", "ute")}
    return {
        "flashmask_weights": {"q": bf(1, 4, 20, 64), "k": bf(1, 2, 20, 64), "lse": floats(1, 4, 20), **bounds, "scale": 0.1},
        "flashmask_cache_weights": {"q": bf(1, 4, 3, 64), **pool, "lse": floats(1, 4, 3), "scale": 0.1, "before": floats(1, 2, 32),
                                    "out": floats(1, 2, 32)},
        "flashmask_cache_evict": {**pool, "weights": floats(1, 2, 32), "new_table": ints(1, 1), "keep": 16},
        "flashmask_decode_tree": {"q": bf(1, 4, 3, 64), **pool, "parents": ints(1, 3), "scale": 0.1},
        "flashmask_cache_accept": {"pools": [bf(6, 2, 16, 64)], "table": ints(1, 2), "lens": ints(1), "T": 3, "path": ints(1, 2)}}


@pytest.mark.parametrize("entry", list(_tensors("cpu")))
def test_tensors_on_the_host_are_refused(entry):
    with pytest.raises(fm.FlashMaskError):
        getattr(fm, entry)(**_tensors("cpu")[entry])


@pytest.mark.gpu
@pytest.mark.parametrize("entry", list(_tensors("cpu")))
def test_each_wrong_tensor_is_refused(entry):
    call, args = getattr(fm, entry), _tensors("cuda")[entry]
    call(**args)
    for name, t in args.items():
        if not isinstance(t, torch.Tensor):
            continue
        other = torch.int64 if t.dtype == torch.int32 else torch.float64
        strided = torch.zeros((*t.shape[:-1], 2 * t.shape[-1]), dtype=t.dtype, device="cuda")[..., ::2]
        wrongs = [t.cpu(), t.to(other), t.reshape(-1)[0], t[None]]
        if t.shape[-1] > 1:
            wrongs.append(strided)
        if t.shape[-1] != 32 or entry == "flashmask_cache_weights":      # weights of any number of places will do
            wrongs.append(torch.cat((t, t)))
        for wrong in wrongs:
            if name in ("k_cache", "v_cache") and wrong.dim() == 4 and wrong.shape[0] == 12:
                wrong = wrong[:, :1]
            with pytest.raises(fm.FlashMaskError):
                call(**(args | {name: wrong}))
    torch.cuda.synchronize()


@pytest.mark.gpu
def test_wrong_numbers_are_refused():
    t = _tensors("cuda")
    for entry, wrong in (("flashmask_weights", {"first_row": 20}), ("flashmask_weights", {"first_row": -1}), ("flashmask_weights", {"first_row": BEYOND}),
                         ("flashmask_weights", {"scale": 0.0}), ("flashmask_cache_weights", {"decay": -1.0}), ("flashmask_cache_weights", {"window": -1}),
                         ("flashmask_cache_weights", {"bounds": t["flashmask_decode_tree"]["table"]}), ("flashmask_cache_evict", {"keep": 0}),
                         ("flashmask_cache_evict", {"keep": 33}), ("flashmask_cache_evict", {"keep": BEYOND + 16}), ("flashmask_cache_evict", {"first": 17}),
                         ("flashmask_cache_evict", {"recent": BEYOND}), ("flashmask_decode_tree", {"window": -1}), ("flashmask_decode_tree", {"scale": -1.0}),
                         ("flashmask_cache_accept", {"T": 0}), ("flashmask_cache_accept", {"T": BEYOND + 3}), ("flashmask_cache_accept", {"T": 1}),
                         ("flashmask_cache_accept", {"pools": []}),
                         ("flashmask_cache_accept", {"pools": [torch.zeros((6, 2, 16, 64), dtype=x, device="cuda") for x in (torch.bfloat16, torch.float16)]})):
        with pytest.raises(fm.FlashMaskError):
            getattr(fm, entry)(**(t[entry] | wrong))
    torch.cuda.synchronize()


@pytest.mark.gpu
def test_windows_of_any_size():
    """A window beyond every length hides nothing."""
    t = _tensors("cuda")
    gen = torch.Generator(device="cuda").manual_seed(1)
    for name in ("flashmask_cache_weights", "flashmask_decode_tree"):
        args = t[name]
        for x in ("q", "k_cache", "v_cache"):
            args[x] = torch.randn(args[x].shape, device="cuda", generator=gen).bfloat16()
        args["lens"], args["table"] = torch.full_like(args["lens"], 30), torch.tensor([[1, 4]], dtype=torch.int32, device="cuda")
        first = [x.clone() for x in getattr(fm, name)(**args)]
        for window in (30, 1 << 30, (1 << 31) - 1, BEYOND + 5):
            assert all(torch.equal(a, b) for a, b in zip(getattr(fm, name)(**args, window=window), first)), window
        assert not all(torch.equal(a, b) for a, b in zip(getattr(fm, name)(**args, window=4), first))
