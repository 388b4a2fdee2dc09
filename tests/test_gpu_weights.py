"""GPU: flashmask_weights against the definition in 64 bits."""
import numpy as np
import pytest
import torch

from keys_util import check_weights, ints
from oracle import keys_oracle as orc
from serving_util import f64, strided

pytestmark = pytest.mark.gpu


def _bounds(kind, B, N, rng):
    at = np.arange(N)
    out = []
    for b in range(B):
        lts, lte, uts, ute = np.full(N, N), np.full(N, N), np.zeros(N, int), at.copy()
        if kind == "full":
            ute = np.zeros(N, int)
        elif kind == "window":
            lts = np.minimum(at + 37, N)
        elif kind == "docs":
            ends = np.append(np.sort(rng.integers(1, max(N, 2), 4)), N)
            lts = ends[np.searchsorted(ends, at, side="right").clip(max=4)]
        elif kind == "both_ways":       # and a last part whose rows and keys see nothing
            cut, pad = N // 3, N - N // 5
            lts = np.where(at < cut, cut, pad)
            ute = np.where(at < cut, 0, cut)
            lts[pad:], ute[pad:] = 0, N
        elif kind == "random":
            lts, lte, uts, ute = rng.integers(-3, N + 3, (4, N))
        elif kind == "nothing":
            lts = np.zeros(N, int)
        out.append((lts, lte, uts, ute))
    return tuple(np.stack(x) for x in zip(*out))


def _problem(seed, B, H, Hk, N, d, kind, packed=False):
    """q, k, lse, bounds; lse from the definition, as the attention call gives it."""
    rng = np.random.default_rng(seed)
    gen = torch.Generator(device="cuda").manual_seed(seed)
    q, k = (strided(torch.randn((B, h, N, d), device="cuda", generator=gen).bfloat16(), packed) for h in (H, Hk))
    bounds = _bounds(kind, B, N, rng)
    i, j = np.arange(N)[:, None], np.arange(N)
    lse = np.zeros((B, H, N))
    for b in range(B):
        lts, lte, uts, ute = (x[b] for x in bounds)
        seen = ~(((lts <= i) & (i < lte)) | ((uts <= i) & (i < ute)))
        for h in range(H):
            s = np.where(seen, f64(q[b, h]) @ f64(k[b, h // (H // Hk)]).T * d ** -0.5, -np.inf)
            top = s.max(1)
            top = np.where(np.isneginf(top), 0, top)
            with np.errstate(divide="ignore"):
                lse[b, h] = top + np.log(np.exp(s - top[:, None]).sum(1))
    return q, k, torch.tensor(lse, dtype=torch.float32, device="cuda"), bounds


def _check(problem, first_row=0, what=""):
    import paper_2410_01359_amd as fm
    q, k, lse, bounds = problem
    d = q.shape[-1]
    got = fm.flashmask_weights(q, k, lse, *(ints(x) for x in bounds), d ** -0.5, first_row=first_row)
    assert got.dtype == torch.float32 and got.shape == (k.shape[0], k.shape[1], k.shape[2])
    want = orc.weights(f64(q), f64(k), f64(lse), bounds, d ** -0.5, first_row)
    check_weights(got, *want, d, what)
    return got


CASES = [
    # B, H, Hk, N, d
    (1, 1, 1, 1, 64), (2, 2, 1, 2, 128), (1, 4, 2, 63, 64), (1, 3, 3, 64, 128), (2, 5, 1, 65, 128), (1, 8, 2, 255, 64), (1, 2, 2, 257, 128),
    (3, 6, 3, 333, 64), (1, 40, 8, 520, 128), (2, 4, 4, 1030, 64), (1, 2, 1, 2049, 128),
]


@pytest.mark.parametrize("kind", ["causal", "full", "window", "docs", "both_ways", "random", "nothing"])
@pytest.mark.parametrize("case", range(len(CASES)))
def test_against_the_definition(case, kind):
    B, H, Hk, N, d = CASES[case]
    got = _check(_problem(case, B, H, Hk, N, d, kind, packed=case % 2 == 1))
    if kind == "nothing":
        assert (got == 0).all()


@pytest.mark.parametrize("case,first_row", [(0, 0), (2, 62), (3, 63), (4, 1), (5, 200), (7, 269), (8, 500), (9, 7), (10, 1985), (10, 100)])
@pytest.mark.parametrize("kind", ["causal", "docs", "random"])
def test_last_rows(kind, case, first_row):
    B, H, Hk, N, d = CASES[case]
    _check(_problem(50 + case, B, H, Hk, N, d, kind, packed=case % 2 == 0), first_row)


def test_hidden_values_have_no_influence():
    """Keys that no row sees and rows that see nothing hold NaN and infinities; a key that some rows see is a number for those alone."""
    q, k, lse, bounds = _problem(7, 1, 2, 1, 300, 64, "both_ways")
    pad = 300 - 60
    k[:, :, pad:] = torch.nan
    q[:, :, pad + 1::2], q[:, :, pad::2] = torch.inf, torch.nan
    import paper_2410_01359_amd as fm
    got = fm.flashmask_weights(q, k, lse, *(ints(x) for x in bounds), 64 ** -0.5)
    want = orc.weights(f64(torch.where(torch.isfinite(q), q, 0)), f64(torch.where(torch.isfinite(k), k, 0)), f64(lse), bounds, 64 ** -0.5)
    check_weights(got, *want, 64)
    assert (got[:, :, pad:] == 0).all()


def test_after_the_attention_call():
    """Every row that sees something gives its keys 1 in all: lse of the forward itself."""
    import paper_2410_01359_amd as fm
    B, H, Hk, N, d = 2, 8, 2, 1500, 128
    q, k, _, bounds = _problem(9, B, H, Hk, N, d, "docs", packed=True)
    v = torch.randn_like(k)
    bounds = tuple(ints(x) for x in bounds)
    _, lse = fm.flashmask_fwd_ex(q, k, v, *bounds, d ** -0.5)
    got = fm.flashmask_weights(q, k, lse, *bounds, d ** -0.5)
    # lse is off by 2e-5 at most at this size: products, sums and logarithm in 32 bits
    assert abs(float(got.double().sum()) - B * H * N) <= B * H * N * 4e-5


def test_strides_and_the_same_bits():
    """A slice of a packed projection, rows apart, an axis of size 1 of any stride; the same call twice, and on another stream."""
    import paper_2410_01359_amd as fm
    gen = torch.Generator(device="cuda").manual_seed(3)
    N, H, Hk, d = 700, 8, 2, 64
    qkv = torch.randn((1, N, H + 2 * Hk, d), device="cuda", generator=gen).bfloat16()
    q, k = qkv[:, :, :H].transpose(1, 2), qkv[:, :, H:H + Hk].transpose(1, 2)
    _, _, _, bounds = _problem(1, 1, 1, 1, N, d, "causal")
    bounds = tuple(ints(x) for x in bounds)
    lse = torch.randn((1, H, N), device="cuda", generator=gen) + 6
    got = fm.flashmask_weights(q, k, lse, *bounds, 0.125)
    check_weights(got, *orc.weights(f64(q), f64(k), f64(lse), [x.cpu().numpy() for x in bounds], 0.125), d)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        again = fm.flashmask_weights(q.contiguous(), k.contiguous(), lse, *bounds, 0.125)
    side.synchronize()
    assert torch.equal(got, again)


def test_graph():
    """Captured and replayed with eager calls of other sizes between, a workspace of its own."""
    import paper_2410_01359_amd as fm
    q, k, lse, bounds = _problem(11, 1, 4, 2, 900, 64, "causal")
    bounds = tuple(ints(x) for x in bounds)
    other = _problem(12, 1, 2, 2, 200, 128, "full")
    ws = torch.empty(fm.flashmask_weights_workspace_bytes(1, 4, 2, 900, 64), dtype=torch.uint8, device="cuda")
    want = fm.flashmask_weights(q, k, lse, *bounds, 0.125)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        got = fm.flashmask_weights(q, k, lse, *bounds, 0.125, workspace=ws)
    for _ in range(3):
        got.fill_(-1)
        ws.fill_(255)
        graph.replay()
        fm.flashmask_weights(other[0], other[1], other[2], *(ints(x) for x in other[3]), 0.1)
        torch.cuda.synchronize()
        assert torch.equal(got, want)
