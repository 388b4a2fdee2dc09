"""GPU: the operators on weights, eviction and trees on several streams at once, each call with what it allocates itself, give the bits that they give alone."""
import pytest
import torch

from keys_util import ints, paged, queries

pytestmark = pytest.mark.gpu


def _calls(seed, T):
    import paper_2410_01359_amd as fm
    lens = [900 + 40 * seed, 300, 64 + seed]
    p = paged(seed, lens, 2, 16, 64, "bf16", spare=40)
    q = queries(seed, 3, 8, T, 64, "bf16")
    pool = (p["k_cache"], p["v_cache"], p["table"], p["lens"])
    lse = torch.full((3, 8, T), 6.0, device="cuda")
    spare = torch.arange(p["k_cache"].shape[0], device="cuda")
    spare = spare[~torch.isin(spare, p["table"].long())][:24].to(torch.int32).view(3, 8).contiguous()
    N = 500 + seed
    prompt = [queries(seed + 1, 1, h, N, 64, "bf16") for h in (4, 2)]
    at = torch.arange(N, dtype=torch.int32, device="cuda")[None].contiguous()
    bounds = (torch.full_like(at, N), torch.full_like(at, N), torch.zeros_like(at), at)
    rows = torch.full((1, 4, N), 6.0, device="cuda")
    parents = ints([[t - 1 if t % 4 else t // 2 - 1 for t in range(T)]] * 3)

    def run():
        tree = fm.flashmask_decode_tree(q, *pool, parents, 0.125)
        weights = fm.flashmask_cache_weights(q, *pool, lse, 0.125)
        table, lens, after, kept = fm.flashmask_cache_evict(*pool, weights, spare, 100, first=4, recent=30)
        pools = [x.clone() for x in pool[:2]]
        lens = fm.flashmask_cache_accept(pools, table, lens, T, ints([[1, 3, -1]] * 3))
        return (*tree, weights, table, lens, after, kept, fm.flashmask_weights(*prompt, rows, *bounds, 0.125), *[x.view(torch.int16) for x in pools])
    return run


@pytest.mark.parametrize("T", [6, 30])
def test_streams_at_once(T):
    calls = [_calls(seed, T) for seed in range(4)]
    want = [[x.clone() for x in call()] for call in calls]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in calls]
    got = []
    for _ in range(3):
        for stream, call in zip(streams, calls):
            with torch.cuda.stream(stream):
                got.append(call())
    torch.cuda.synchronize()
    for i, results in enumerate(got):
        assert all(torch.equal(a, b) for a, b in zip(results, want[i % len(calls)])), i
