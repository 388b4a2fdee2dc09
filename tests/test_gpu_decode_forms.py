"""GPU: forms of flashmask_decode in pairs: a window together with bounds, more than 8 new tokens in every pair of types, both masks in every pair
of types, and a stream of its own."""
import numpy as np
import pytest
import torch

from test_gpu_decode import CASES, _check, _problem, _reference

pytestmark = pytest.mark.gpu

PAIRS = [("bf16", "bf16"), ("f16", "f16"), ("bf16", "e4m3"), ("f16", "e4m3")]


@pytest.mark.parametrize("type,cache", PAIRS)
@pytest.mark.parametrize("case", [1, 4, 5, 8, 10, 11])
def test_window_and_bounds(case, type, cache):
    lens, H, Hk, T, d, page, columns = CASES[case]
    a = _problem(600 + case, lens, H, Hk, T, d, page, type, cache, packed=case % 2 == 1, columns=columns, mask="bounds")
    for window in (1, 50, 600):
        a["window"] = window
        _check(a, type, what=f"window {window} ")


@pytest.mark.parametrize("type,cache", [("f16", "f16"), ("bf16", "e4m3")])
@pytest.mark.parametrize("mask", ["window", "bounds"])
@pytest.mark.parametrize("case", [2, 7, 8, 11])
def test_masks_of_the_other_types(case, mask, type, cache):
    lens, H, Hk, T, d, page, columns = CASES[case]
    _check(_problem(700 + case, lens, H, Hk, T, d, page, type, cache, packed=case % 2 == 0, columns=columns, mask=mask), type)


@pytest.mark.parametrize("type,cache", PAIRS)
@pytest.mark.parametrize("mask", ["none", "window", "bounds"])
@pytest.mark.parametrize("lens,H,Hk,T,d,columns", [([40, 700, 9], 4, 2, 17, 128, None), ([330], 6, 2, 100, 64, None), ([260, 2600], 8, 1, 33, 128, 200),
                                                   ([4200], 1, 1, 256, 64, None)])
def test_many_new_tokens(lens, H, Hk, T, d, columns, mask, type, cache):
    _check(_problem(800 + T, lens, H, Hk, T, d, 16, type, cache, columns=columns, mask=mask), type)


def test_on_a_stream_of_its_own():
    """The launches of a split call go to the current stream, behind what made its inputs there and before what reads its results."""
    import paper_2410_01359_amd as fm
    a = _problem(900, [1500, 2100, 0, 77], 8, 2, 2, 128, 16, "bf16", "bf16")
    want = fm.flashmask_decode(**a)
    torch.cuda.synchronize()
    stream = torch.cuda.Stream()
    busy = torch.randn((4096, 4096), device="cuda")
    with torch.cuda.stream(stream):
        for _ in range(20):
            busy = busy @ busy * 1e-3
        q = torch.zeros_like(a["q"])
        q.copy_(a["q"])
        out, lse = fm.flashmask_decode(**(a | {"q": q}))
        got = out.clone(), lse.clone()
    stream.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(got, want))


def test_window_of_one_sees_the_row_itself():
    """Values come out as they are, wherever the sequence is cut."""
    import paper_2410_01359_amd as fm
    a = _problem(901, [1, 16, 17, 1300], 4, 4, 1, 64, 16, "bf16", "bf16", columns=100)
    a["window"] = 1
    out, _ = fm.flashmask_decode(**a)
    for b, n in enumerate((1, 16, 17, 1300)):
        page = int(a["table"][b, (n - 1) // 16])
        assert torch.equal(out[b, :, 0], a["v_cache"][page, :, (n - 1) % 16])
    assert np.isfinite(_reference(a)[1]).all()
