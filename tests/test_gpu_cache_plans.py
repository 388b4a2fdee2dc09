"""GPU: lists of free pages and compactions on both sides of the lines between page maps in LDS and in global memory."""
import numpy as np
import pytest
import torch

from serving_util import orc

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("num_pages", [(1 << 16) - 1, 1 << 16, 1 << 17, (1 << 17) + 1])
@pytest.mark.parametrize("entries", [1 << 17, (1 << 17) + 1])
def test_large_tables(num_pages, entries):
    import paper_2410_01359_amd as fm
    rng = np.random.default_rng(num_pages + entries)
    named = rng.permutation(num_pages)[:num_pages // 2]
    table = rng.choice(named, size=(1, entries)).astype(np.int32)
    table[rng.random(table.shape) < 0.2] = -1
    table[0, -1] = named[0]
    device = torch.tensor(table, device="cuda")
    used = np.unique(table[table >= 0])                     # the definition, without the oracle's loops over pages
    free, count = fm.flashmask_cache_free_list(device, num_pages)
    assert int(count) == num_pages - len(used)
    assert np.array_equal(free.cpu().numpy()[:num_pages - len(used)], np.setdiff1d(np.arange(num_pages), used)) and (free[num_pages - len(used):] == -1).all()
    to = np.arange(num_pages)
    to[used[used >= len(used)]] = np.setdiff1d(np.arange(len(used)), used)
    pool = torch.zeros((num_pages, 1, 16, 64), device="cuda", dtype=torch.uint8)
    pool[:, 0, 0, :4] = torch.arange(num_pages, device="cuda", dtype=torch.int32).view(torch.uint8).view(-1, 4)
    got_table, got_used = fm.flashmask_cache_compact([pool], device)
    assert int(got_used) == len(used) and np.array_equal(got_table.cpu().numpy(), np.where(table >= 0, to[table], -1))
    held = pool[:, 0, 0, :4].contiguous().view(torch.int32).view(-1).cpu().numpy()
    assert np.array_equal(held[to[used]], used)


def test_table_of_many_entries_and_few_pages():
    import paper_2410_01359_amd as fm
    table = np.random.default_rng(1).integers(-1, 300, size=(1000, 1001)).astype(np.int32)
    table[table == 17] = 18
    free, count = fm.flashmask_cache_free_list(torch.tensor(table, device="cuda"), 310)
    want, n = orc.free_list(table, 310)
    assert int(count) == n == 11 and np.array_equal(free.cpu().numpy(), want)
