"""GPU: flashmask_weights of prompts with more row tiles than are listed together (2048): what is carried from one list to the next, against the definition in
64 bits."""
import numpy as np
import pytest
import torch

from keys_util import check_weights

pytestmark = pytest.mark.gpu

N = 131072 + 37 + 701       # 701 rows behind the first list of the rows from 37 on


def _bounds(kind):
    at = np.arange(N)
    lts, lte, uts, ute = np.full(N, N), np.full(N, N), np.zeros(N, int), at.copy()
    if kind == "window":
        lts = np.minimum(at + 300, N)
    elif kind == "docs":        # one of them over the seam
        ends = np.array([1000, 40007, 130500, 131500, N])
        lts = ends[np.searchsorted(ends, at, side="right")]
    elif kind == "full":
        ute = np.zeros(N, int)
    return [torch.tensor(x, dtype=torch.int32, device="cuda")[None] for x in (lts, lte, uts, ute)]


def _definition(q, k, bounds, scale, first_row):
    """lse of the rows that count [H, N]; of a single K/V head the weights, the same of terms times their size, and the number of terms."""
    H, d = q.shape[1], q.shape[3]
    k = k[0, 0].double()
    kt, kt_abs = k.T.contiguous(), k.abs().T.contiguous()
    lts, lte, uts, ute = (x[0] for x in bounds)
    lse = torch.zeros((H, N), dtype=torch.float32, device="cuda")
    out, size, terms = (torch.zeros(N, dtype=torch.float64, device="cuda") for _ in range(3))
    step = 1024
    for begin in range(first_row, N, step):
        i = torch.arange(begin, min(begin + step, N), device="cuda")[:, None]
        seen = ~(((lts <= i) & (i < lte)) | ((uts <= i) & (i < ute)))
        for h in range(H):
            rows = q[0, h, begin:begin + step].double()
            s = torch.where(seen, rows @ kt * scale, -torch.inf)
            lse[h, begin:begin + step] = s.logsumexp(1)
            back = lse[h, begin:begin + step, None].double()
            p = (s - back).exp_()
            out += p.sum(0)
            size += (p * ((rows.abs() @ kt_abs) * scale + back.abs())).sum(0)
            terms += seen.sum(0)
    return lse, [x.cpu().numpy()[None, None] for x in (out, size, terms)]


@pytest.mark.parametrize("kind", ["causal", "window", "docs", "full"])
@pytest.mark.parametrize("H,d,first_row", [(1, 64, 37), (2, 128, 37)])
def test_against_the_definition(H, d, first_row, kind):
    import paper_2410_01359_amd as fm
    gen = torch.Generator(device="cuda").manual_seed(d)
    q, k = (torch.randn((1, h, N, d), device="cuda", generator=gen).bfloat16() for h in (H, 1))
    bounds, scale = _bounds(kind), d ** -0.5
    lse, want = _definition(q, k, bounds, scale, first_row)
    got = fm.flashmask_weights(q, k, lse[None], *bounds, scale, first_row=first_row)
    check_weights(got, *want, d)
    # of the rows behind the seam alone, too
    _, want = _definition(q, k, bounds, scale, N - 701)
    check_weights(fm.flashmask_weights(q, k, lse[None], *bounds, scale, first_row=N - 701), *want, d)
