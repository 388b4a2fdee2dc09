"""GPU: examples/generate.py, which uses the operators around the attention call together: a step over the cache gives what the
whole sequence gives without one, after forks and a compaction, and a training step's gradients are those of the layer in 64 bits."""
import importlib.util
import os

import numpy as np
import pytest
import torch

from oracle import cache_oracle, flashmask_oracle as orc
from serving_util import f64

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def _example():
    spec = importlib.util.spec_from_file_location("generate", os.path.join(ROOT, "examples", "generate.py"))
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


@pytest.mark.parametrize("type,cache,bar", [
    # out, and keys, queries and P of the call without a cache, are rounded to 8 bits (bf16): a few of those of the largest output
    (torch.bfloat16, torch.bfloat16, 8 * 2.0 ** -8),
    (torch.float16, torch.float16, 8 * 2.0 ** -8),
    # keys and values are off by up to 2^-4 of themselves, an output by an average of that over few keys and by what the scores (of size
    # one) change in the weights
    (torch.bfloat16, torch.float8_e4m3fn, 4 * 2.0 ** -4),
])
def test_steps_over_the_cache(type, cache, bar):
    assert _example().generate(type, cache, steps=24) <= bar


@pytest.mark.parametrize("way,size", [("speculate", {"rounds": 4}), ("speculate", {"rounds": 3, "drafted": 70}), ("forget", {"steps": 70}),
                                      ("forget", {"steps": 30, "prompt": 119, "most": 130, "keep": 128})])
@pytest.mark.parametrize("type,cache,bar", [
    # as above
    (torch.bfloat16, torch.bfloat16, 8 * 2.0 ** -8),
    (torch.float16, torch.float16, 8 * 2.0 ** -8),
    (torch.bfloat16, torch.float8_e4m3fn, 4 * 2.0 ** -4),
])
def test_trees_and_eviction(type, cache, bar, way, size):
    assert getattr(_example(), way)(type, cache, **size) <= bar


def test_training_step():
    example = _example()
    layer = example.Layer(torch.bfloat16, torch.bfloat16, 1)
    gen = torch.Generator(device="cuda").manual_seed(7)
    N, H, Hk, d = 45, example.HEADS, example.KV_HEADS, example.D
    x = torch.randn((1, N, example.MODEL), device="cuda", generator=gen).bfloat16()
    dout = torch.randn((1, H, N, d), device="cuda", generator=gen).bfloat16()
    got = example.train_step(layer, x, dout)
    q, k, v = (f64(y.transpose(1, 2))[0] for y in layer.project(x))
    freqs, at = example.FREQS.numpy(), np.arange(N)
    rq, rk = (cache_oracle.rope(y, at, freqs, False) for y in (q, k))
    bounds = (np.full(N, N), np.full(N, N), np.zeros(N, int), np.arange(N))
    drq, drk, dv = orc.backward_grouped(rq, rk, v, f64(dout)[0], *bounds, d ** -0.5)[:3]
    want = (cache_oracle.rope(drq, at, freqs, False, backward=True), cache_oracle.rope(drk, at, freqs, False, backward=True), dv)
    for name, g, w in zip("qkv", got, want):
        assert np.abs(f64(g)[0] - w).max() <= 5e-2 * max(1.0, np.abs(w).max() / 4), name
