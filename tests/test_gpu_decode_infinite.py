"""GPU: an infinite value that a row sees comes out as itself however little weight its key has, as long as the weight is a normal number of 32
bits, and takes nothing from the other elements."""
import math

import numpy as np
import pytest
import torch

from serving_util import TYPES

pytestmark = pytest.mark.gpu


def _ints(x):
    return torch.tensor(np.asarray(x), dtype=torch.int32, device="cuda")


@pytest.mark.parametrize("columns", [20, 100])                     # one launch, and chunks that a second one joins
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("length,at,top", [(2, 1, 0), (2, 0, 1), (300, 7, 299), (300, 290, 12), (300, 131, 132)])
@pytest.mark.parametrize("type", ["bf16", "f16"])
def test_far_below_the_maximum(type, length, at, top, d, columns):
    """Weights of 2^-8 to 2^-120; the keys beside the two have scores another 100 below."""
    import paper_2410_01359_amd as fm
    pages = -(-length // 16)
    gaps = torch.tensor([8, 24, 27, 38, 39, 40, 41, 60, 80, 100, 110, 111, 112, 113, 115, 118, 120.0])
    B = len(gaps)
    k, v = torch.zeros((B * pages * 16, d)), torch.ones((B * pages * 16, d))
    for b, gap in enumerate(gaps):
        row = b * pages * 16
        k[row:row + pages * 16, 0] = -220.0
        k[row + at, 0], k[row + top, 0] = -gap, 0.0
        v[row + at, 3], v[row + at, 4], v[row + top, 5] = math.inf, -math.inf, math.nan
    k, v = (x.view(B * pages, 1, 16, d).cuda().to(TYPES[type]) for x in (k, v))
    q = torch.zeros((B, 1, 1, d), device="cuda", dtype=TYPES[type])
    q[..., 0] = 1
    table = np.full((B, columns), -1)
    table[:, :pages] = np.arange(B * pages).reshape(B, pages)
    out, lse = fm.flashmask_decode(q, k, v, _ints(table), _ints([length] * B), math.log(2))
    out = out[:, 0, 0].float().cpu()
    assert (out[:, 3] == math.inf).all() and (out[:, 4] == -math.inf).all(), [(float(g), x) for g, x in zip(gaps, out[:, 3:5].tolist())]
    assert out[:, 5].isnan().all()
    assert ((out[:, 6:] - 1).abs() <= torch.finfo(TYPES[type]).eps / 2).all() and ((out[:, :3] - 1).abs() <= torch.finfo(TYPES[type]).eps / 2).all()
    assert ((lse[:, 0, 0].cpu().double() - torch.log1p(2.0 ** -gaps.double())).abs() <= 2.0 ** -20).all()
