"""One attention layer generating text-like sequences with the library: the operators around the attention call, used together.

    python examples/generate.py [--way steps|trees|forget] [--type bf16|f16] [--e4m3] [--steps N]

Random weights, random token embeddings.  Prompts are written to a paged cache and attended to by flashmask_fwd_ex; each
step then rotates and writes one new token per sequence (flashmask_cache_append) and attends to the cache (flashmask_decode).
Half way, every sequence is forked into two that go on differently, some sequences end, and the cache is compacted.  At the
end each sequence's last outputs are computed again from scratch, without a cache, and compared.
`speculate` drafts trees of tokens instead, attends to all of a tree in one call (flashmask_decode_tree) and takes a path of it over
(flashmask_cache_accept).  `forget` sums up what attention weight every key gets (flashmask_weights for the prompt, flashmask_cache_weights for
each step) and drops the light ones when a sequence has become too long (flashmask_cache_evict).
`train_step` is the same layer's share of a training step: rotation, attention, and the gradients of both.
"""
from __future__ import annotations

import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2410_01359_amd as fm  # noqa: E402

HEADS, KV_HEADS, D, PAGE, MODEL = 8, 2, 64, 16, 256
FREQS = 10000.0 ** (-torch.arange(0, D, 2, dtype=torch.float64) / D)


def causal_bounds(B, N):
    """LTS, LTE, UTS, UTE of a causal mask."""
    at = torch.arange(N, dtype=torch.int32, device="cuda").expand(B, N).contiguous()
    return torch.full_like(at, N), torch.full_like(at, N), torch.zeros_like(at), at


class Layer:
    """Projections of one attention layer and the cache of its sequences."""

    def __init__(self, dtype, cache_dtype, pages, seed=0):
        gen = torch.Generator(device="cuda").manual_seed(seed)
        self.dtype = dtype
        self.qkv = (torch.randn((MODEL, (HEADS + 2 * KV_HEADS) * D), device="cuda", generator=gen) / MODEL ** 0.5).to(dtype)
        self.freqs = FREQS.cuda()
        self.pools = [torch.zeros((pages, KV_HEADS, PAGE, D), device="cuda").to(cache_dtype) for _ in range(2)]
        self.scales = {}
        if cache_dtype == torch.float8_e4m3fn:
            self.scales = {n: torch.full((KV_HEADS,), 0.02, device="cuda") for n in ("k_scale", "v_scale")}

    def project(self, x):
        """q [..., H, d], k, v [..., H_kv, d] of embeddings x."""
        return (x @ self.qkv).unflatten(-1, (HEADS + 2 * KV_HEADS, D)).split((HEADS, KV_HEADS, KV_HEADS), dim=-2)

    def append(self, x, table, seqs, positions):
        """Writes the tokens x [n, MODEL] to the cache; their rotated queries."""
        q, k, v = self.project(x)
        return fm.flashmask_cache_append(k, v, *self.pools, table, seqs, positions, q=q, freqs=self.freqs, **self.scales)

    def write(self, x, table, positions, places):
        """Writes the tokens x [B, T, MODEL], which are at `positions` [B, T] of their sequences, to other places; their rotated queries."""
        q, k, v = (y.transpose(1, 2) for y in self.project(x))
        q, k = fm.flashmask_rope(q, k, self.freqs, positions=positions)
        seqs = torch.arange(len(x), dtype=torch.int32, device="cuda").repeat_interleave(x.shape[1])
        fm.flashmask_cache_append(*(y.transpose(1, 2).flatten(0, 1) for y in (k, v)), *self.pools, table, seqs, places.flatten(), **self.scales)
        return q

    def decode(self, q, table, lens):
        return fm.flashmask_decode(q[:, :, None], *self.pools, table, lens, D ** -0.5, **self.scales)[0][:, :, 0]

    def full(self, x):
        """Outputs [B, H, N, d] of whole sequences x [B, N, MODEL], without the cache (bf16)."""
        q, k, v = (y.bfloat16().transpose(1, 2) for y in self.project(x))
        q, k = fm.flashmask_rope(q, k, self.freqs)
        return fm.flashmask_fwd_ex(q, k, v, *causal_bounds(x.shape[0], x.shape[1]), D ** -0.5)[0]


def train_step(layer, x, dout):
    """Gradients of the projections' outputs q, k, v (bf16) for upstream gradients dout [B, H, N, d]."""
    q, k, v = (y.bfloat16().transpose(1, 2) for y in layer.project(x))
    rq, rk = fm.flashmask_rope(q, k, layer.freqs)
    bounds = causal_bounds(x.shape[0], x.shape[1])
    out, lse = fm.flashmask_fwd_ex(rq, rk, v, *bounds, D ** -0.5)
    drq, drk, dv = fm.flashmask_bwd_ex(rq, rk, v, out, lse, dout, *bounds, D ** -0.5)
    dq, dk = fm.flashmask_rope_bwd(drq, drk, layer.freqs)
    return dq, dk, dv


def generate(dtype=torch.bfloat16, cache_dtype=None, steps=40, prompts=(1, 17, 90, 33), pages=128):
    """Largest difference between the outputs of the last step and those computed from scratch, relative to the largest output."""
    layer = Layer(dtype, cache_dtype or dtype, pages)
    gen = torch.Generator(device="cuda").manual_seed(1)

    def embeddings(n):
        return torch.randn((n, MODEL), device="cuda", generator=gen).to(dtype)

    def ints(x):
        return torch.tensor(x, dtype=torch.int32, device="cuda")

    columns = -(-(max(prompts) + steps) // PAGE)
    free = list(range(pages))
    rows = [[free.pop() for _ in range(-(-n // PAGE))] for n in prompts]
    lens = list(prompts)

    def tables():
        return ints([r + [-1] * (columns - len(r)) for r in rows])

    # the prompts, all tokens in one call
    texts = [embeddings(n) for n in prompts]
    layer.append(torch.cat(texts), tables(), ints([b for b, n in enumerate(prompts) for _ in range(n)]),
                 ints([j for n in prompts for j in range(n)]))
    out = None
    for step in range(steps):
        if step == steps // 2:
            # every sequence goes on as two; the second one needs its own copy of a last page that is not full
            B = len(rows)
            new = [-1] * B + [free.pop() if n % PAGE else -1 for n in lens]
            table, lengths = fm.flashmask_cache_fork(layer.pools, tables(), ints(lens), ints(list(range(B)) * 2), ints(new), PAGE)
            rows = [[p for p in r if p >= 0] for r in table.tolist()]
            lens, texts = lengths.tolist(), texts * 2
            # the first sequence ends, and the pages in use move to the front
            rows, lens, texts = rows[1:], lens[1:], texts[1:]
            table, used = fm.flashmask_cache_compact(layer.pools, tables())
            rows = [[p for p in r if p >= 0] for r in table.tolist()]
            listed, count = fm.flashmask_cache_free_list(table, pages)
            free = listed[:int(count)].tolist()
            assert int(used) + len(free) == pages
        for r, n in zip(rows, lens):
            if n % PAGE == 0:
                r.append(free.pop())
        x = embeddings(len(rows))
        table = tables()
        q = layer.append(x, table, ints(list(range(len(rows)))), ints(lens))
        lens = [n + 1 for n in lens]
        texts = [torch.cat((t, x[b:b + 1])) for b, t in enumerate(texts)]
        out = layer.decode(q, table, ints(lens))
    worst = 0.0
    for b, text in enumerate(texts):
        want = layer.full(text[None])[0, :, -1].float()
        worst = max(worst, float((out[b].float() - want).abs().max() / want.abs().max()))
    return worst


def speculate(dtype=torch.bfloat16, cache_dtype=None, rounds=6, drafted=13, prompts=(1, 17, 90, 33)):
    """Largest difference between the outputs of accepted tokens and those computed from scratch, relative to the largest output."""
    columns = -(-(max(prompts) + rounds * drafted) // PAGE)
    B, T, pages = len(prompts), drafted, len(prompts) * columns
    layer, rng = Layer(dtype, cache_dtype or dtype, pages), torch.Generator().manual_seed(3)
    gen = torch.Generator(device="cuda").manual_seed(2)
    table = torch.randperm(pages, generator=rng).to(torch.int32).view(B, columns).cuda()
    texts = [torch.randn((n, MODEL), device="cuda", generator=gen).to(dtype) for n in prompts]
    for b, text in enumerate(texts):
        at = torch.arange(len(text), dtype=torch.int32, device="cuda")
        layer.append(text, table, torch.full_like(at, b), at)
    lens, worst = torch.tensor(prompts, dtype=torch.int32, device="cuda"), 0.0
    for _ in range(rounds):
        # a random tree; a real program has the tokens that a small model thinks likely
        parents = torch.stack([torch.cat([torch.randint(-1, t, (1,), generator=rng) if t else torch.tensor([-1]) for t in range(T)]) for _ in range(B)])
        depth, path = torch.zeros((B, T), dtype=torch.int32), torch.full((B, T), -1, dtype=torch.int32)
        for b in range(B):
            for t in range(T):
                depth[b, t] = depth[b, parents[b, t]] + 1 if parents[b, t] >= 0 else 0
            t, n = -1, 0       # accepted: any way down; a real program goes by the outputs
            while len(children := (parents[b] == t).nonzero().flatten()):
                t = int(children[torch.randint(len(children), (1,), generator=rng)])
                path[b, n], n = t, n + 1
        x = torch.randn((B, T, MODEL), device="cuda", generator=gen).to(dtype)
        places = lens[:, None] + torch.arange(T, dtype=torch.int32, device="cuda")
        q = layer.write(x, table, lens[:, None] + depth.cuda(), places)
        out, _ = fm.flashmask_decode_tree(q, *layer.pools, table, lens + T, parents.to(torch.int32).cuda(), D ** -0.5, **layer.scales)
        lens = fm.flashmask_cache_accept(layer.pools, table, lens + T, T, path.cuda())
        for b in range(B):
            way = path[b][path[b] >= 0].long().cuda()
            texts[b] = torch.cat((texts[b], x[b, way]))
            assert len(texts[b]) == int(lens[b])
            want = layer.full(texts[b][None])[0, :, -len(way):].float()
            worst = max(worst, float((out[b][:, way].float() - want).abs().max() / want.abs().max()))
    return worst


def forget(dtype=torch.bfloat16, cache_dtype=None, steps=40, prompt=100, most=120, keep=64, sequences=3):
    """Largest difference between the outputs of the last step and attention over the kept tokens' own keys and values, relative to the
    largest output."""
    columns, B = -(-max(most, prompt + 1) // PAGE), sequences
    layer, gen = Layer(dtype, cache_dtype or dtype, 2 * B * columns), torch.Generator(device="cuda").manual_seed(4)
    table, spare = torch.randperm(2 * B * columns, device="cuda", generator=gen).to(torch.int32).view(2, B, columns).unbind()
    table, spare = table.contiguous(), spare.contiguous()
    text = torch.randn((B, prompt, MODEL), device="cuda", generator=gen).to(dtype)

    def places(n):
        return torch.arange(n, dtype=torch.int32, device="cuda").repeat(B, 1)

    # the prompt: what its last rows look at is what counts
    layer.write(text, table, places(prompt), places(prompt))
    q, k, v = (y.bfloat16().transpose(1, 2) for y in layer.project(text))
    q, k = fm.flashmask_rope(q, k, layer.freqs)
    bounds = causal_bounds(B, prompt)
    _, lse = fm.flashmask_fwd_ex(q, k, v, *bounds, D ** -0.5)
    weights = torch.zeros((B, KV_HEADS, columns * PAGE), device="cuda")
    weights[:, :, :prompt] = fm.flashmask_weights(q, k, lse, *bounds, D ** -0.5, first_row=max(prompt - 32, 0))
    lens = torch.full((B,), prompt, dtype=torch.int32, device="cuda")
    # which token of the text a place has
    who = torch.arange(columns * PAGE, device="cuda").expand(B, KV_HEADS, -1).clone()
    for _ in range(steps):
        if int(lens.max()) == most:
            new, lens, weights, kept = fm.flashmask_cache_evict(*layer.pools, table, lens, weights, spare, keep, first=4, recent=16, **layer.scales)
            who[:, :, :keep] = who.gather(2, kept.long())
            assert torch.equal(new[:, :keep // PAGE], spare[:, :keep // PAGE])
            table, spare = spare, table        # the old pages are free
        x = torch.randn((B, 1, MODEL), device="cuda", generator=gen).to(dtype)
        who.scatter_(2, lens.long()[:, None, None].expand(B, KV_HEADS, 1), text.shape[1])
        q = layer.write(x, table, torch.full((B, 1), text.shape[1], dtype=torch.int32, device="cuda"), lens[:, None])
        text, lens = torch.cat((text, x), 1), lens + 1
        out, lse = fm.flashmask_decode(q, *layer.pools, table, lens, D ** -0.5, **layer.scales)
        weights = fm.flashmask_cache_weights(q, *layer.pools, table, lens, lse, D ** -0.5, weights, decay=0.95, **layer.scales)
    _, k, v = (y.transpose(1, 2) for y in layer.project(text))
    _, k = fm.flashmask_rope(k, k, layer.freqs)
    n = int(lens[0])
    k, v = (y.float().gather(2, who[:, :, :n, None].expand(-1, -1, -1, D)).repeat_interleave(HEADS // KV_HEADS, 1) for y in (k, v))
    want = torch.softmax(q.float() @ k.transpose(2, 3).contiguous() * D ** -0.5, -1) @ v
    return float((out.float() - want).abs().max() / want.abs().max())


def main():
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    ap.add_argument("--type", choices=("bf16", "f16"), default="bf16")
    ap.add_argument("--e4m3", action="store_true", help="8-bit cache")
    ap.add_argument("--steps", type=int, default=40)
    ap.add_argument("--way", choices=("steps", "trees", "forget"), default="steps")
    a = ap.parse_args()
    dtype = torch.bfloat16 if a.type == "bf16" else torch.float16
    cache = torch.float8_e4m3fn if a.e4m3 else dtype
    if a.way != "steps":
        off = speculate(dtype, cache, a.steps) if a.way == "trees" else forget(dtype, cache, a.steps)
        print(f"{a.steps} {a.way}: outputs differ from those without a cache by {off:.4f} of the largest")
        return
    off = generate(dtype, cache, a.steps)
    print(f"{a.steps} steps: last outputs differ from those without a cache by {off:.4f} of the largest")
    layer = Layer(torch.bfloat16, torch.bfloat16, 1)
    x = torch.randn((2, 500, MODEL), device="cuda").bfloat16()
    grads = train_step(layer, x, torch.randn((2, HEADS, 500, D), device="cuda").bfloat16())
    print("training step: gradients", ", ".join(f"{n} {list(g.shape)}" for n, g in zip(("q", "k", "v"), grads)))


if __name__ == "__main__":
    main()
