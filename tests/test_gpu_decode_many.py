"""GPU: flashmask_decode of hundreds to thousands of sequences, whose chunks a launch of their own lists."""
import numpy as np
import pytest
import torch

from test_gpu_decode import _check, _ints, _problem

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("mask", ["none", "window"])
@pytest.mark.parametrize("B,H,Hk,T,long,type,cache", [(257, 16, 16, 1, 1300, "bf16", "bf16"), (600, 6, 3, 1, 1100, "f16", "e4m3"),
                                                      (1024, 4, 4, 1, 1500, "bf16", "bf16"), (1025, 2, 2, 2, 2000, "bf16", "e4m3"), (2200, 2, 1, 1, 1100, "f16", "f16")])
def test_against_the_definition(B, H, Hk, T, long, type, cache, mask):
    """Short sequences, empty ones, and long ones that are split on either side of a round of 1024."""
    lens = np.random.default_rng(B).integers(0, 12, size=B)
    lens[[0, B // 2, min(1023, B - 1), B - 1]] = long, long // 2, long - 1, long - 300
    _check(_problem(500 + B, lens, H, Hk, T, 64, 16, type, cache, mask=mask), type)


def test_no_keys_at_all():
    import paper_2410_01359_amd as fm
    B = 700
    cache = torch.full((1, 8, 16, 64), torch.nan, device="cuda", dtype=torch.bfloat16)
    q = torch.ones((B, 8, 1, 64), device="cuda", dtype=torch.bfloat16)
    lens = _ints(np.arange(B) % 3 * -5)
    out, lse = fm.flashmask_decode(q, cache, cache, _ints(np.full((B, 80), -1)), lens, 0.125)
    assert (out == 0).all() and lse.isneginf().all()


def test_graph_replays():
    """The list is made again by every replay, from the lengths as they are then."""
    import paper_2410_01359_amd as fm
    rng = np.random.default_rng(3)
    B, heads, d, columns = 400, 8, 64, 80
    gen = torch.Generator(device="cuda").manual_seed(3)
    cache = [torch.randn((200, heads, 16, d), device="cuda", generator=gen).bfloat16() for _ in range(2)]
    q = torch.randn((B, heads, 1, d), device="cuda", generator=gen).bfloat16()
    table, lens = _ints(rng.integers(0, 200, size=(B, columns))), _ints(rng.integers(0, 60, size=B))
    ws = torch.full((fm.flashmask_decode_workspace_bytes(B, heads, heads, 1, d),), 255, dtype=torch.uint8, device="cuda")
    fm.flashmask_decode(q, *cache, table, lens, 0.125, workspace=ws)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = fm.flashmask_decode(q, *cache, table, lens, 0.125, workspace=ws)
    for trial in range(4):
        lens.copy_(_ints(np.where(rng.random(B) < 0.1, rng.integers(0, columns * 16 + 9, size=B), rng.integers(0, 30, size=B))))
        eager = [x.clone() for x in fm.flashmask_decode(q, *cache, table, lens, 0.125)]
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(eager, captured)), trial


def test_setup_does_not_grow_with_the_square_of_the_sequences():
    """8192 short sequences in rows of the table that may hold long ones (whose calls are split) take little more than in short rows (which are
    not): it was eleven times as much when every workgroup went over all lengths."""
    import paper_2410_01359_amd as fm
    B, heads, d = 8192, 8, 64
    gen = torch.Generator(device="cuda").manual_seed(4)
    cache = [torch.randn((3 * 64, heads, 16, d), device="cuda", generator=gen).bfloat16() for _ in range(2)]
    q = torch.randn((B, heads, 1, d), device="cuda", generator=gen).bfloat16()
    lens = torch.randint(1, 41, (B,), device="cuda", generator=gen, dtype=torch.int32)
    short = torch.randint(0, 192, (B, 3), device="cuda", generator=gen, dtype=torch.int32)
    long = torch.nn.functional.pad(short, (0, 69), value=-1)
    ws = torch.empty(fm.flashmask_decode_workspace_bytes(B, heads, heads, 1, d), dtype=torch.uint8, device="cuda")
    times = {}
    for name, table in (("short", short), ("long", long)):
        start, end = (torch.cuda.Event(enable_timing=True) for _ in range(2))
        best = float("inf")
        for _ in range(6):
            start.record()
            out = fm.flashmask_decode(q, *cache, table, lens, 0.125, workspace=ws)
            end.record()
            torch.cuda.synchronize()
            best = min(best, start.elapsed_time(end))
        times[name] = best, out
    assert torch.equal(times["short"][1][0], times["long"][1][0])
    assert times["long"][0] < 3 * times["short"][0], {n: t for n, (t, _) in times.items()}
