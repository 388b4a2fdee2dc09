"""GPU: flashmask_cache_append, _fork, _free_list and _compact against their definitions."""
import numpy as np
import pytest
import torch

from serving_util import TYPES, cache_of, check, f64, orc, raw, rounding, strided

pytestmark = pytest.mark.gpu


def _frequencies(rot):
    return torch.tensor(10000.0 ** (-2.0 * np.arange(rot // 2) / rot), device="cuda")


def _ints(*x):
    return torch.tensor(np.array(*x), dtype=torch.int32, device="cuda")


@pytest.mark.parametrize("type,cache", [("bf16", "bf16"), ("f16", "f16"), ("bf16", "e4m3"), ("f16", "e4m3")])
@pytest.mark.parametrize("tokens,H,Hk,d,page,rot,interleaved,packed", [
    (1, 1, 1, 64, 16, 64, False, False),
    (45, 4, 2, 128, 48, 128, True, True),
    (70, 6, 3, 64, 16, 32, False, True),
    (300, 8, 1, 128, 64, 48, True, False),
    (9, 0, 2, 128, 32, 0, False, False),
    (50, 64, 8, 128, 16, 128, False, True),
    (700, 16, 16, 64, 32, 64, True, False),
])
def test_append(tokens, H, Hk, d, page, rot, interleaved, packed, type, cache):
    import paper_2410_01359_amd as fm
    rng = np.random.default_rng(tokens)
    gen = torch.Generator(device="cuda").manual_seed(tokens)
    sequences, columns = 5, -(-2 * tokens // page) + 1
    num_pages = sequences * columns + 2
    table = rng.permutation(num_pages)[:sequences * columns].reshape(sequences, columns).astype(np.int32)
    # every token its own place; padding, positions beyond the row and below 0, rows without that page and with pages that are none
    places = rng.permutation(sequences * columns * page)[:tokens]
    seqs, positions = places // (columns * page), places % (columns * page)
    if tokens > 8:
        table[1, 0], table[2, -1], table[3, 1] = -1, num_pages, np.iinfo(np.int32).max
        seqs[:4] = (-1, sequences, np.iinfo(np.int32).min, np.iinfo(np.int32).max)
        positions[4:8] = (-1, columns * page, np.iinfo(np.int32).max, np.iinfo(np.int32).min)
    qkv = torch.randn((tokens, H + 2 * Hk, d), device="cuda", generator=gen).to(TYPES[type])
    if tokens > 8:
        qkv[8, -1, 3], qkv[8, -1, 4] = 3000.0, -3000.0    # beyond the 8-bit type
    q, k, v = qkv[:, :H], qkv[:, H:H + Hk], qkv[:, H + Hk:]
    caches = [cache_of(gen, cache, num_pages, Hk, page, d, packed) for _ in range(2)]
    scales = [torch.rand(Hk, device="cuda", generator=gen) + 0.5 for _ in range(2)] if cache == "e4m3" else [None, None]
    before = [f64(c) for c in caches]
    freqs = _frequencies(rot) if rot else None
    got = fm.flashmask_cache_append(k, v, *caches, _ints(table), _ints(seqs), _ints(positions), q=q if H else None, freqs=freqs,
                                    layout=fm.FM_ROPE_INTERLEAVED if interleaved else fm.FM_ROPE_HALF, amp=1.5, k_scale=scales[0], v_scale=scales[1])

    def turned(x):
        x = f64(x)
        return orc.rope(x, positions[:, None], freqs.cpu().numpy(), interleaved, 1.5) if rot else x

    def slack(x):   # of the rotation in 32 bits: the pair's size is at most both elements'
        return 8 * 2.0 ** -24 * 1.5 * 2 * np.abs(x).max(-1, keepdims=True) if rot else 0 * np.abs(x)

    if H:
        check(f64(got), turned(q), rounding(type, turned(q)) * (1 + 2.0 ** -20) + slack(f64(q)), "q")
    else:
        assert got is None
    for name, c, x, old, scale in (("k", caches[0], turned(k), before[0], scales[0]), ("v", caches[1], f64(v), before[1], scales[1])):
        s = 1.0 if scale is None else f64(scale)[:, None]
        rows = np.clip(x / s, -448, 448) if scale is not None else x
        off = rounding(cache, rows) * (1 + 2.0 ** -20) + ((slack(x) / s if name == "k" else 0 * rows) + 2.0 ** -23 * np.abs(rows) if scale is not None
                                                           else slack(x) if name == "k" else 0 * rows)
        ref = orc.append(old, rows, table, page, seqs, positions)
        bound = orc.append(np.zeros_like(old), np.broadcast_to(off, rows.shape), table, page, seqs, positions)
        check(f64(c), ref, bound, name)


def test_append_of_every_8_bit_value_is_exact():
    """All finite values of the 8-bit type, and values half way between neighbours, which go to the even one."""
    import paper_2410_01359_amd as fm
    codes = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).float()
    codes = codes[codes.isfinite()].sort().values
    x = torch.cat((codes, (codes[1:] + codes[:-1]) / 2))
    x = torch.nn.functional.pad(x, (0, 512 - x.numel())).view(4, 1, 128).to(torch.float16).cuda()
    cache = [torch.zeros((1, 1, 16, 128), device="cuda").to(torch.float8_e4m3fn) for _ in range(2)]
    one = torch.ones(1, device="cuda")
    fm.flashmask_cache_append(x, x, *cache, _ints([[0]]), _ints([0] * 4), _ints(range(4)), k_scale=one, v_scale=one)
    want = x[:, 0].float().to(torch.float8_e4m3fn).float()
    for c in cache:
        assert torch.equal(c[0, 0, :4].float(), want)
    x[0, 0, :3] = torch.tensor([torch.nan, torch.inf, -torch.inf])
    fm.flashmask_cache_append(x, x, *cache, _ints([[0]]), _ints([0] * 4), _ints(range(4)), k_scale=one, v_scale=one)
    assert cache[0][0, 0, 0, 0].float().isnan() and cache[0][0, 0, 0, 1:3].float().tolist() == [448.0, -448.0]


@pytest.mark.parametrize("cache", ["bf16", "e4m3"])
@pytest.mark.parametrize("pools,page,heads,d,packed", [(1, 16, 1, 64, False), (2, 64, 4, 128, False), (5, 48, 3, 64, True), (130, 16, 1, 64, False)])
def test_fork(pools, page, heads, d, packed, cache):
    import paper_2410_01359_amd as fm
    gen = torch.Generator(device="cuda").manual_seed(page)
    B, columns, num_pages = 6, 4, 40
    lens = np.array([0, 1, page, 2 * page + 5, 4 * page, 3 * page - 1], np.int32)
    order = np.random.default_rng(page).permutation(num_pages)
    table = np.full((B, columns), -1, np.int32)
    taken = 0
    for b in range(B):
        n = -(-lens[b] // page)
        table[b, :n] = order[taken:taken + n]
        taken += n
    parents = np.array([3, 3, 3, 1, 0, 4, 5, 2, -1, 6, 5, 1], np.int32)
    new = np.array([-1, *order[taken:taken + 8], -1, num_pages, -5], np.int32)
    stored = [cache_of(gen, cache, num_pages, heads, page, d, packed) for _ in range(pools)]
    want_pools, want_table, want_lens = orc.fork([raw(p).cpu().numpy() for p in stored], table, lens, parents, new, page)
    got_table, got_lens = fm.flashmask_cache_fork(stored, _ints(table), _ints(lens), _ints(parents), _ints(new), page)
    assert np.array_equal(got_table.cpu().numpy(), want_table) and np.array_equal(got_lens.cpu().numpy(), want_lens)
    for got, want in zip(stored, want_pools):
        assert np.array_equal(raw(got).cpu().numpy(), want)


def test_fork_with_lengths_and_rows_that_name_no_page():
    import paper_2410_01359_amd as fm
    pool = torch.arange(4.0, device="cuda").view(4, 1, 1, 1).expand(4, 1, 16, 64).contiguous().bfloat16()
    table = np.array([[9, -1], [-1, 1 << 30], [0, 1]], np.int32)
    lens, parents, new = np.array([5, 20, 1 << 30], np.int32), np.array([0, 1, 2], np.int32), np.array([1, 2, 3], np.int32)
    want = orc.fork([f64(pool)], table, lens, parents, new, 16)
    got = fm.flashmask_cache_fork([pool], _ints(table), _ints(lens), _ints(parents), _ints(new), 16)
    assert np.array_equal(got[0].cpu().numpy(), want[1]) and np.array_equal(f64(pool), want[0][0])


@pytest.mark.parametrize("num_pages,shape,share", [(1, (1, 1), 1.0), (33, (3, 4), 0.5), (100, (7, 20), 0.3), (1000, (16, 100), 0.9), (4096, (40, 64), 0.5),
                                                   (5000, (300, 1000), 0.2), (140000, (64, 1000), 0.4)])
def test_free_list_and_compact(num_pages, shape, share):
    """Up to tables and page counts that go through global memory."""
    import paper_2410_01359_amd as fm
    rng = np.random.default_rng(num_pages)
    named = rng.permutation(num_pages)[:max(1, int(share * num_pages))]
    table = rng.choice(named, size=shape).astype(np.int32)             # shared pages, and some that nobody names
    table[rng.random(shape) < 0.2] = -1
    table[rng.random(shape) < 0.01] = num_pages
    gen = torch.Generator(device="cuda").manual_seed(num_pages)
    pools = [cache_of(gen, "bf16", num_pages, 1, 16, 64) for _ in range(1 if num_pages > 5000 else 70 if num_pages == 100 else 2)]
    want_free, want_count = orc.free_list(table, num_pages)
    free, count = fm.flashmask_cache_free_list(_ints(table), num_pages)
    assert int(count) == want_count and np.array_equal(free.cpu().numpy(), want_free)
    want_pools, want_table, want_used = orc.compact([raw(p).cpu().numpy() for p in pools], table)
    got_table, used = fm.flashmask_cache_compact(pools, _ints(table))
    assert int(used) == want_used and np.array_equal(got_table.cpu().numpy(), want_table)
    for got, want in zip(pools, want_pools):
        assert np.array_equal(raw(got).cpu().numpy(), want)


@pytest.mark.parametrize("entry", [-1, 0])
def test_tables_of_one_value(entry):
    import paper_2410_01359_amd as fm
    table, pool = _ints([[entry] * 5]), torch.zeros((7, 2, 16, 64), device="cuda", dtype=torch.bfloat16)
    free, count = fm.flashmask_cache_free_list(table, 7)
    assert int(count) == 7 - (entry == 0) and free.tolist() == (list(range(7)) if entry < 0 else [1, 2, 3, 4, 5, 6, -1])
    got, used = fm.flashmask_cache_compact([pool], table)
    assert torch.equal(got, table) and int(used) == (entry == 0)


def test_refusals():
    import paper_2410_01359_amd as fm
    kv = torch.zeros((3, 2, 64), device="cuda", dtype=torch.bfloat16)
    cache = torch.zeros((4, 2, 16, 64), device="cuda", dtype=torch.bfloat16)
    eight, scale = cache.to(torch.float8_e4m3fn), torch.ones(2, device="cuda")
    table, three, freqs = _ints([[0, 1]]), _ints([0, 0, 0]), _frequencies(64)
    at = _ints([0, 1, 2])
    fm.flashmask_cache_append(kv, kv, cache, cache.clone(), table, three, at, q=kv, freqs=freqs)
    ok = {"k": kv, "v": kv, "k_cache": cache, "v_cache": cache, "table": table, "seqs": three, "positions": at}
    for wrong in ({"k": kv.half(), "v": kv.half()}, {"v": kv.half()}, {"k": kv[:2]}, {"v": kv[:, :1]}, {"k": kv.float(), "v": kv.float()}, {"k": kv.cpu()},
                  {"k_cache": cache[:3]}, {"v_cache": cache.half()}, {"k_cache": cache.float(), "v_cache": cache.float()},
                  {"k_cache": cache[:, :, :8], "v_cache": cache[:, :, :8]}, {"k_cache": cache[..., :32], "v_cache": cache[..., :32]},
                  {"k_cache": cache[:, :1], "v_cache": cache[:, :1]}, {"k_cache": cache[:0], "v_cache": cache[:0]},
                  {"k_cache": cache[:, :1].expand(4, 2, 16, 64)},
                  {"k_cache": eight, "v_cache": eight}, {"k_scale": scale, "v_scale": scale}, {"k_cache": eight, "v_cache": eight, "k_scale": scale},
                  {"k_cache": eight, "v_cache": eight, "k_scale": scale[:1], "v_scale": scale}, {"table": table.long()}, {"table": table[0]},
                  {"table": table.cpu()}, {"seqs": three[:2]}, {"seqs": three.long()}, {"positions": at.float()}, {"q": kv}, {"q": kv[:2], "freqs": freqs},
                  {"q": kv.half(), "freqs": freqs}, {"freqs": freqs.float()}, {"freqs": freqs[:0]}, {"freqs": freqs[:4]}, {"freqs": freqs, "layout": 5},
                  {"freqs": freqs, "amp": float("nan")}):
        with pytest.raises(fm.FlashMaskError):
            fm.flashmask_cache_append(**(ok | wrong))
    one = _ints([0])
    fm.flashmask_cache_fork([cache], table, one, one, one, 16)
    other = torch.zeros((4, 2, 16, 128), device="cuda", dtype=torch.bfloat16)
    for wrong in ([], [cache, other], [cache, cache.half()], [other[..., :64]], [cache.cpu()], [cache[:, :, ::2]], [strided(cache, True), cache]):
        with pytest.raises(fm.FlashMaskError):
            fm.flashmask_cache_fork(wrong, table, one, one, one, 16)
        with pytest.raises(fm.FlashMaskError):
            fm.flashmask_cache_compact(wrong, table)
    for wrong in ((table[0], one, one, one, 16), (table.long(), one, one, one, 16), (table, at, one, one, 16), (table, one, one, at, 16),
                  (table, one, one[:0], one[:0], 16), (table, one, one, one, 0), (table, one.cpu(), one, one, 16)):
        with pytest.raises(fm.FlashMaskError):
            fm.flashmask_cache_fork([cache], *wrong)
    small = torch.empty(256, dtype=torch.uint8, device="cuda")
    for call in (lambda: fm.flashmask_cache_free_list(table, 0), lambda: fm.flashmask_cache_free_list(table.long(), 4),
                 lambda: fm.flashmask_cache_free_list(table[:, :0], 4), lambda: fm.flashmask_cache_free_list(table, 4000, workspace=small),
                 lambda: fm.flashmask_cache_compact([cache], table[:0]), lambda: fm.flashmask_cache_compact([cache], table.cpu())):
        with pytest.raises(fm.FlashMaskError):
            call()
    torch.cuda.synchronize()
