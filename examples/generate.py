"""One attention layer generating text-like sequences with the library: the operators around the attention call, used together.

    python examples/generate.py [--type bf16|f16] [--e4m3] [--steps N]

Random weights, random token embeddings.  Prompts are written to a paged cache and attended to by flashmask_fwd_ex; each
step then rotates and writes one new token per sequence (flashmask_cache_append) and attends to the cache (flashmask_decode).
Half way, every sequence is forked into two that go on differently, some sequences end, and the cache is compacted.  At the
end each sequence's last outputs are computed again from scratch, without a cache, and compared.
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


def main():
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    ap.add_argument("--type", choices=("bf16", "f16"), default="bf16")
    ap.add_argument("--e4m3", action="store_true", help="8-bit cache")
    ap.add_argument("--steps", type=int, default=40)
    a = ap.parse_args()
    dtype = torch.bfloat16 if a.type == "bf16" else torch.float16
    off = generate(dtype, torch.float8_e4m3fn if a.e4m3 else dtype, a.steps)
    print(f"{a.steps} steps: last outputs differ from those without a cache by {off:.4f} of the largest")
    layer = Layer(torch.bfloat16, torch.bfloat16, 1)
    x = torch.randn((2, 500, MODEL), device="cuda").bfloat16()
    grads = train_step(layer, x, torch.randn((2, HEADS, 500, D), device="cuda").bfloat16())
    print("training step: gradients", ", ".join(f"{n} {list(g.shape)}" for n, g in zip(("q", "k", "v"), grads)))


if __name__ == "__main__":
    main()
