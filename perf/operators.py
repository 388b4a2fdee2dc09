"""Performance cases of the operators around the attention call: rotary positions, writing new tokens to a paged
key-value cache, attention of new tokens over that cache, forking and compacting its pages.

A case is one pass of what a training or serving program has them do.  `own` selects the library's entry points; without it
the same outputs come from elementary torch operations.  The cases run from one short sequence (nothing but latency) to
131072 cached tokens and gigabytes of pages, over both head dimensions, the types and layouts that the entry points
take, odd lengths, empty sequences and padding tokens.

Fields of a case, by kind:
  kind     "rope"    q, k rotated forward, the gradients of both rotated back (a training step's share)
           "append"  new tokens rotated and written to the cache; a token with sequence -1 is padding
           "decode"  T new tokens of each sequence attend to the cache
           "fork"    children of sequences: rows of the page table, the last page copied where it is not full
           "reclaim" after sequences ended: list of free pages, and the cache compacted to its front
  B, H, Hk, N, T, d, page   sequences, query and K/V heads, (longest) length, new tokens, head dimension, tokens to a page
  type, cache               element types; an e4m3 cache has a scale for each K/V head
  packed                    tensors stored [B,N,H,d] and caches [pages,page,Hk,d], passed as strided views
  len_seed                  draws lengths, documents and parents, which belong to the case (the tensors to the seed)
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

_TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16, "e4m3": torch.float8_e4m3fn}
_SIZE = {"f32": 4, "bf16": 2, "f16": 2, "e4m3": 1}


def _rope(name, B, H, Hk, N, d, type, rot, interleaved, docs, packed, stretch=1.0, len_seed=3):
    return {"name": name, "kind": "rope", "B": B, "H": H, "Hk": Hk, "N": N, "d": d, "type": type, "rot": rot,
            "interleaved": interleaved, "docs": docs, "packed": packed, "stretch": stretch, "len_seed": len_seed}


def _append(name, B, H, Hk, N, d, page, type, cache, rot, interleaved, prompt, packed=False, len_seed=3):
    return {"name": name, "kind": "append", "B": B, "H": H, "Hk": Hk, "N": N, "d": d, "page": page, "type": type,
            "cache": cache, "rot": rot, "interleaved": interleaved, "prompt": prompt, "packed": packed, "len_seed": len_seed}


def _decode(name, B, H, Hk, N, T, d, page, type, cache, mask="none", packed=False, ragged=False, len_seed=3):
    return {"name": name, "kind": "decode", "B": B, "H": H, "Hk": Hk, "N": N, "T": T, "d": d, "page": page, "type": type,
            "cache": cache, "mask": mask, "packed": packed, "ragged": ragged, "len_seed": len_seed}


def _fork(name, B, children, Hk, N, d, page, cache, pools, len_seed=3):
    return {"name": name, "kind": "fork", "B": B, "children": children, "Hk": Hk, "N": N, "d": d, "page": page,
            "cache": cache, "pools": pools, "len_seed": len_seed}


def _reclaim(name, B, Hk, N, d, page, cache, pools, len_seed=3):
    return {"name": name, "kind": "reclaim", "B": B, "Hk": Hk, "N": N, "d": d, "page": page, "cache": cache,
            "pools": pools, "len_seed": len_seed}


def listed():
    return [
        # the smallest training call, a part of the head in the interleaved layout, positions 0 to N - 1
        _rope("rope_part_500", 1, 2, 2, 500, 64, "f32", 32, True, 0, False),
        # long-context training on packed documents, grouped heads, projections stored [B,N,H,d], stretched positions
        _rope("rope_docs_32768", 1, 32, 8, 32768, 128, "bf16", 128, False, 34, True, 4.0),
        # one decoding step of 48 sequences, three of them padding
        _append("append_step_48", 48, 32, 8, 2048, 128, 64, "bf16", "bf16", 128, False, False),
        # the prompts of five requests, of odd lengths, into an 8-bit cache of small pages
        _append("append_prompts_e4m3", 5, 32, 8, 4099, 128, 16, "bf16", "e4m3", 64, True, True),
        # the smallest decoding call: one short sequence, nothing but latency
        _decode("decode_333", 1, 8, 8, 333, 1, 128, 16, "bf16", "bf16"),
        # continuous batching: 64 sequences of very different lengths, an empty one and one of a single token among them
        _decode("decode_ragged_8192", 64, 32, 8, 8192, 1, 128, 64, "bf16", "bf16", ragged=True),
        # one sequence of 131072 tokens: all of the chip on eight K/V heads
        _decode("decode_long_131072", 1, 32, 8, 131072, 1, 128, 256, "bf16", "bf16"),
        # four drafted tokens to be verified, questions with several answers, 8-bit cache stored [pages,page,Hk,d]
        _decode("verify_answers_e4m3", 16, 32, 4, 16384, 4, 64, 32, "f16", "e4m3", "answers", packed=True, ragged=True),
        # eight requests of four beams each choose their parents, one layer
        _fork("fork_beams_32", 32, 32, 8, 1000, 128, 64, "bf16", 2),
        # 64 prompts sampled four times each, six layers
        _fork("fork_samples_256", 64, 256, 8, 2048, 128, 64, "bf16", 12),
        # a small cache after half of its sequences ended
        _reclaim("reclaim_small", 16, 4, 700, 64, 16, "bf16", 2),
        # a large one, six layers
        _reclaim("reclaim_layers", 128, 8, 4096, 128, 64, "bf16", 12),
    ]


_MOST_BYTES = 1.3e9   # no drawn case moves more than the largest listed one


def draw(rng):
    def spread(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    while True:
        kind = rng.choice(("rope", "append", "decode", "decode", "decode", "fork", "reclaim"))
        d = rng.choice((64, 128, 128))
        Hk = rng.choice((1, 2, 4, 8, 8, 16))
        H = Hk * rng.choice((1, 2, 4, 5, 8))
        seed = rng.randint(0, 1 << 30)
        page = rng.choice((16, 32, 64, 128, 256))
        type = rng.choice(("bf16", "bf16", "f16"))
        cache = rng.choice((type, type, "e4m3"))
        packed = rng.random() < 0.4
        if kind == "rope":
            rot = rng.choice((d, d, d // 2, d // 4))
            case = _rope("", rng.choice((1, 1, 2, 4)), H, Hk, spread(200, 131072), d, rng.choice((type, type, "f32")), rot,
                         rng.random() < 0.5, rng.randint(0, 12), packed, rng.choice((1.0, 1.0, 8.0)), seed)
        elif kind == "append":
            prompt = rng.random() < 0.5
            B = rng.randint(1, 8) if prompt else spread(1, 256)
            case = _append("", B, H, Hk, spread(64, 16384), d, page, type, cache, rng.choice((d, d, d // 2)),
                           rng.random() < 0.5, prompt, packed, seed)
        elif kind == "decode":
            case = _decode("", spread(1, 128), H, Hk, spread(64, 131072), rng.choice((1, 1, 1, 2, 5, 8)), d, page, type, cache,
                           rng.choice(("none", "none", "window", "answers")), packed, rng.random() < 0.7, seed)
        elif kind == "fork":
            B = spread(1, 64)
            case = _fork("", B, B * rng.choice((1, 2, 4)), Hk, spread(100, 4096), d, page, cache, rng.choice((2, 4, 12)), seed)
        else:
            case = _reclaim("", spread(4, 256), Hk, spread(100, 8192), d, page, cache, rng.choice((2, 4, 12)), seed)
        del case["name"]
        if work(case)["bytes"] <= _MOST_BYTES and _held(case) <= 12e9:
            return case


# --- what belongs to a case: lengths, documents, parents, which sequences ended
def _lengths(case):
    """Tokens of each sequence; the longest has N.  A ragged batch has an empty and a one-token sequence in it."""
    B, N = case["B"], case["N"]
    rng = np.random.default_rng([case["len_seed"], 1])
    if not case.get("ragged", True):
        return np.full(B, N, np.int64)
    lens = np.exp(rng.uniform(math.log(max(1, N // 64)), math.log(N + 1), size=B)).astype(np.int64).clip(1, N)
    lens[0] = N
    if case["kind"] == "decode" and B >= 8:
        lens[3], lens[5] = 0, 1
    return lens


def _pages(case):
    """Pages of each sequence."""
    return -(-_lengths(case) // case["page"])


def _prompt_lengths(case):
    return _lengths(case) if case["prompt"] else np.ones(case["B"], np.int64)


def _answers(case):
    """Bounds of questions (two fifths) with three answers that do not see each other; the new tokens go on with the third."""
    lens, N = _lengths(case), case["N"]
    lts = np.full((case["B"], N), N, np.int64)
    for row, L in enumerate(lens):
        question, L = int(L) * 2 // 5, int(L)
        ends = question + (L - question) * np.arange(4) // 3
        lts[row, question:ends[1]] = ends[1]
        lts[row, ends[1]:ends[2]] = ends[2]
    return lts


_WINDOW = 1024


def _visible(case):
    """Keys that at least one of a sequence's new tokens sees, per sequence."""
    lens, T = _lengths(case), case["T"]
    if case["mask"] == "window":
        return np.minimum(lens, _WINDOW + T - 1)
    if case["mask"] == "answers":
        ends = lens * 2 // 5 + (lens - lens * 2 // 5) * 2 // 3
        return np.minimum(lens, lens * 2 // 5 + lens - ends + T - 1)   # nothing of the first two answers but their last tokens
    return lens


def _parents(case):
    """Parent of each child, and whether it gets a page of its own (the first child of a parent goes on with the parent's)."""
    B, n = case["B"], case["children"]
    rng = np.random.default_rng([case["len_seed"], 2])
    if n > B:
        parents = np.repeat(np.arange(B), n // B)
    else:                                           # groups of four beams choose among themselves
        parents = np.arange(B) // 4 * 4 + rng.integers(0, 4, size=B)
        parents = np.minimum(parents, B - 1)
    first = np.zeros(len(parents), bool)
    first[np.unique(parents, return_index=True)[1]] = True
    return parents, ~first


def _ended(case):
    rng = np.random.default_rng([case["len_seed"], 3])
    ended = rng.random(case["B"]) < 0.45
    ended[0], ended[-1] = False, True
    return ended


def _page_bytes(case):
    return case["page"] * case["Hk"] * case["d"] * _SIZE[case["cache"]]


def _moves(case):
    """Pages that a compaction moves, about the share of used pages that lies behind their count, and all pages."""
    pages, alive = _pages(case), ~_ended(case)
    shared = np.minimum(np.minimum(pages[2::4][:len(pages[3::4])], pages[3::4]), -(-case["N"] // case["page"]) // 2)
    used = int(pages[alive].sum() - shared[alive[3::4] & alive[2::4][:len(shared)]].sum())
    total = int(pages.sum()) + case["B"]
    return used * (total - used) // total, total


def _held(case):
    """Bytes of a state."""
    if case["kind"] in ("fork", "reclaim"):
        return case["pools"] * _page_bytes(case) * (int(_pages(case).sum()) + case.get("children", case["B"]) + 1)
    if case["kind"] == "rope":
        return 4 * case["B"] * case["N"] * (case["H"] + case["Hk"]) * case["d"] * _SIZE[case["type"]]
    plain = 16 * case["B"] * case["N"] * case["Hk"] * case["d"]      # and what the plain form makes of it
    return 2 * _page_bytes(case) * int(_pages(case).sum()) + plain * (case["kind"] == "decode")


def work(case):
    """Each input read once and each output written once."""
    if case["kind"] == "rope":
        B, H, Hk, N, d = (case[k] for k in ("B", "H", "Hk", "N", "d"))
        values = B * (H + Hk) * N * d
        return {"bytes": 2 * (2 * values * _SIZE[case["type"]] + (4 * B * N if case["docs"] else 0)),
                "flops": 2 * 3 * values * case["rot"] // d}
    if case["kind"] == "append":
        n, H, Hk, d = int(_prompt_lengths(case).sum()), case["H"], case["Hk"], case["d"]
        return {"bytes": n * d * (2 * H + 2 * Hk) * _SIZE[case["type"]] + n * d * 2 * Hk * _SIZE[case["cache"]] + 12 * n,
                "flops": 3 * n * (H + Hk) * case["rot"]}
    if case["kind"] == "decode":
        B, H, Hk, T, d = (case[k] for k in ("B", "H", "Hk", "T", "d"))
        seen, lens = _visible(case), _lengths(case)
        moved = 2 * int(seen.sum()) * Hk * d * _SIZE[case["cache"]] + 2 * B * T * H * d * _SIZE[case["type"]] + 4 * B * T * H
        moved += 4 * int((-(-seen // case["page"])).sum()) + 4 * B
        if case["mask"] == "answers":
            moved += 16 * int(lens.sum())
        return {"bytes": moved, "flops": 4 * H * T * d * int(seen.sum())}
    if case["kind"] == "fork":
        parents, copied = _parents(case)
        pages = int((copied & (_lengths(case)[parents] % case["page"] != 0)).sum())
        return {"bytes": 2 * case["pools"] * pages * _page_bytes(case) + 8 * len(parents) * (-(-case["N"] // case["page"])), "flops": 0}
    moved, total = _moves(case)
    return {"bytes": 2 * case["pools"] * moved * _page_bytes(case) + 8 * case["B"] * (-(-case["N"] // case["page"])) + 4 * total, "flops": 0}


# --- inputs
def _frequencies(case):
    i = torch.arange(case["rot"] // 2, dtype=torch.float64, device="cuda")
    return 10000.0 ** (-2.0 * i / case["rot"]) / case.get("stretch", 1.0)


def _pool(case, pages, gen):
    """Pages of one layer's keys or values, indexed [page, head, token, d]."""
    shape = (pages, case["page"], case["Hk"], case["d"]) if case.get("packed") else (pages, case["Hk"], case["page"], case["d"])
    x = torch.randn(shape, device="cuda", dtype=torch.bfloat16, generator=gen).to(_TYPES[case["cache"]])
    return x.transpose(1, 2) if case.get("packed") else x


def _table(case, counts, gen, spare):
    """Page table of sequences with `counts` pages in random order, -1 behind them, and the number of pages."""
    counts = torch.from_numpy(counts).cuda()
    total = int(counts.sum()) + spare
    col = torch.arange(-(-case["N"] // case["page"]), device="cuda")
    order = torch.randperm(total, device="cuda", generator=gen).to(torch.int32)
    at = (counts.cumsum(0) - counts)[:, None] + col
    return torch.where(col < counts[:, None], order[at.clamp(max=total - 1)], -1), order, total


def _scales(case, gen):
    if case["cache"] != "e4m3":
        return None, None
    return tuple(torch.rand(case["Hk"], device="cuda", generator=gen) * 0.5 + 0.75 for _ in range(2))


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    kind = case["kind"]
    state = {"kind": kind}

    def normal(*shape):
        return torch.randn(shape, device="cuda", generator=gen).to(_TYPES[case["type"]])

    if kind == "rope":
        B, N, d = case["B"], case["N"], case["d"]
        for name, heads in (("q", case["H"]), ("k", case["Hk"]), ("dq", case["H"]), ("dk", case["Hk"])):
            state[name] = normal(B, N, heads, d).transpose(1, 2) if case["packed"] else normal(B, heads, N, d)
        state["freqs"] = _frequencies(case)
        state["positions"] = None
        if case["docs"]:     # documents of a packed row, each counted from its own first token
            rng = np.random.default_rng([case["len_seed"], 4])
            starts = np.sort(rng.integers(0, N, size=(B, case["docs"])), axis=1)
            starts[:, 0] = 0
            at = np.arange(N)
            rows = [at - s[np.searchsorted(s, at, side="right") - 1] for s in starts]
            state["positions"] = torch.from_numpy(np.stack(rows).astype(np.int32)).cuda()
        state["interleaved"], state["amp"] = case["interleaved"], 1.0 + 0.1 * math.log(case["stretch"])
        return state

    lens = _lengths(case)
    if kind in ("append", "decode"):
        spare = 3
        table, _, total = _table(case, _pages(case), gen, spare)
        state |= {"table": table, "page": case["page"], "k_cache": _pool(case, total, gen), "v_cache": _pool(case, total, gen)}
        state["k_scale"], state["v_scale"] = _scales(case, gen)
    if kind == "append":
        new = _prompt_lengths(case)
        n, H, Hk, d = int(new.sum()), case["H"], case["Hk"], case["d"]
        qkv = normal(n, H + 2 * Hk, d)            # a packed projection: q, k, v are slices of it
        state |= {"q": qkv[:, :H], "k": qkv[:, H:H + Hk], "v": qkv[:, H + Hk:], "freqs": _frequencies(case), "amp": 1.0,
                  "interleaved": case["interleaved"]}
        seqs = np.repeat(np.arange(case["B"]), new)
        positions = np.concatenate([np.arange(L - c, L) for L, c in zip(lens, new)])
        if not case["prompt"]:
            seqs[7::16] = -1
        state["seqs"], state["positions"] = (torch.from_numpy(x.astype(np.int32)).cuda() for x in (seqs, positions))
    elif kind == "decode":
        B, H, T, d = case["B"], case["H"], case["T"], case["d"]
        state["q"] = normal(B, T, H, d).transpose(1, 2)
        state["lens"] = torch.from_numpy(lens.astype(np.int32)).cuda()
        state["max_len"] = case["N"]
        state["scale"] = 1.0 / math.sqrt(d)
        state["window"] = _WINDOW if case["mask"] == "window" else 0
        state["bounds"] = None
        if case["mask"] == "answers":
            lts = torch.from_numpy(_answers(case).astype(np.int32)).cuda()
            state["bounds"] = (lts, torch.full_like(lts, case["N"]), torch.zeros_like(lts), torch.zeros_like(lts))
        state["scratch"] = torch.zeros(64 << 20, device="cuda", dtype=torch.uint8)   # kept by a serving program
    elif kind == "fork":
        parents, copied = _parents(case)
        table, order, total = _table(case, _pages(case), gen, case["children"])
        new = np.where(copied, total - 1 - np.arange(len(parents)), -1)
        fresh = torch.from_numpy(new).cuda()
        state |= {"table": table, "lens": torch.from_numpy(lens.astype(np.int32)).cuda(), "page": case["page"],
                  "parents": torch.from_numpy(parents.astype(np.int32)).cuda(),
                  "new_pages": torch.where(fresh < 0, -1, order[fresh.clamp(min=0)]),
                  "pools": [_pool(case, total, gen) for _ in range(case["pools"])]}
    else:
        table, _, total = _table(case, _pages(case), gen, case["B"])
        # every fourth sequence shares the first half of its predecessor's pages, as far as both have them
        half = table.shape[1] // 2
        both = (table[3::4, :half] >= 0) & (table[2::4, :half][:table[3::4].shape[0]] >= 0)
        table[3::4, :half] = torch.where(both, table[2::4, :half][:table[3::4].shape[0]], table[3::4, :half])
        table[torch.from_numpy(_ended(case)).cuda()] = -1
        state |= {"table": table, "num_pages": total, "pools": [_pool(case, total, gen) for _ in range(case["pools"])]}
    return state


# --- one pass
def run(state):
    if own:
        return _library(state)
    return {"rope": _plain_rope, "append": _plain_append, "decode": _plain_decode, "fork": _plain_fork,
            "reclaim": _plain_reclaim}[state["kind"]](state)


def _library(state):
    return {"rope": _own_rope, "append": _own_append, "decode": _own_decode, "fork": _own_fork,
            "reclaim": _own_reclaim}[state["kind"]](state)


def _own_rope(s):
    import paper_2410_01359_amd as fm
    how = {"layout": fm.FM_ROPE_INTERLEAVED if s["interleaved"] else fm.FM_ROPE_HALF, "amp": s["amp"]}
    q, k = fm.flashmask_rope(s["q"], s["k"], s["freqs"], s["positions"], **how)
    dq, dk = fm.flashmask_rope_bwd(s["dq"], s["dk"], s["freqs"], s["positions"], **how)
    return q, k, dq, dk


def _own_append(s):
    import paper_2410_01359_amd as fm
    q = fm.flashmask_cache_append(s["k"], s["v"], s["k_cache"], s["v_cache"], s["table"], s["seqs"], s["positions"], q=s["q"],
                                  freqs=s["freqs"], layout=fm.FM_ROPE_INTERLEAVED if s["interleaved"] else fm.FM_ROPE_HALF,
                                  amp=s["amp"], k_scale=s["k_scale"], v_scale=s["v_scale"])
    return q, s["k_cache"], s["v_cache"]


def _own_decode(s):
    import paper_2410_01359_amd as fm
    return fm.flashmask_decode(s["q"], s["k_cache"], s["v_cache"], s["table"], s["lens"], s["scale"], bounds=s["bounds"],
                               window=s["window"], k_scale=s["k_scale"], v_scale=s["v_scale"], workspace=s["scratch"])


def _own_fork(s):
    import paper_2410_01359_amd as fm
    table, lens = fm.flashmask_cache_fork(s["pools"], s["table"], s["lens"], s["parents"], s["new_pages"], s["page"])
    return table, lens, s["pools"]


def _own_reclaim(s):
    import paper_2410_01359_amd as fm
    free, count = fm.flashmask_cache_free_list(s["table"], s["num_pages"])
    table, used = fm.flashmask_cache_compact(s["pools"], s["table"])
    return free, count, table, used, s["pools"]


def _rotated(x, cos, sin, interleaved):
    """x [..., d] in 32 bits, its first elements rotated by the angles whose cosines and sines are given."""
    half = cos.shape[-1]
    head, tail = x[..., :2 * half], x[..., 2 * half:]
    if interleaved:
        a, b = head[..., 0::2], head[..., 1::2]
        return torch.cat((torch.stack((a * cos - b * sin, b * cos + a * sin), -1).flatten(-2), tail), -1)
    a, b = head[..., :half], head[..., half:]
    return torch.cat((a * cos - b * sin, b * cos + a * sin, tail), -1)


def _angles(positions, freqs, amp):
    angle = positions[..., None].double() * freqs          # 64 bits: far positions turn many times
    return (angle.cos() * amp).float(), (angle.sin() * amp).float()


def _plain_rope(s):
    positions = s["positions"]
    if positions is None:
        positions = torch.arange(s["q"].shape[2], device="cuda")[None]
    cos, sin = (x[:, None] for x in _angles(positions, s["freqs"], s["amp"]))
    forward = [_rotated(s[n].float(), cos, sin, s["interleaved"]).to(s[n].dtype) for n in ("q", "k")]
    return *forward, *(_rotated(s[n].float(), cos, -sin, s["interleaved"]).to(s[n].dtype) for n in ("dq", "dk"))


def _plain_append(s):
    cos, sin = (x[:, None] for x in _angles(s["positions"], s["freqs"], s["amp"]))
    q = _rotated(s["q"].float(), cos, sin, s["interleaved"]).to(s["q"].dtype)
    k, v = _rotated(s["k"].float(), cos, sin, s["interleaved"]), s["v"].float()
    if s["k_scale"] is not None:
        k, v = ((x / scale[None, :, None]).clamp(-448, 448) for x, scale in ((k, s["k_scale"]), (v, s["v_scale"])))
    kept = s["seqs"] >= 0
    seqs, at = s["seqs"][kept].long(), s["positions"][kept].long()
    page, slot = s["table"][seqs, at // s["page"]].long(), at % s["page"]
    for x, cache in ((k, s["k_cache"]), (v, s["v_cache"])):
        x = x[kept].to(cache.dtype)
        if x.element_size() == 1:        # values of 8 bits are moved as whole numbers
            x, cache = x.view(torch.uint8), cache.view(torch.uint8)
        cache[page, :, slot] = x
    return q, s["k_cache"], s["v_cache"]


def _plain_decode(s):
    q, table, lens, page, scale = (s[n] for n in ("q", "table", "lens", "page", "scale"))
    B, H, T, d = q.shape
    Hk = s["k_cache"].shape[1]
    j = torch.arange(s["max_len"], device="cuda")
    pages = table[:, j // page]
    at = pages.clamp(min=0).long()

    def cached(cache, factor):       # [B, Hk, keys, d]
        if cache.element_size() == 1:
            x = cache.view(torch.uint8)[at, :, j % page].view(cache.dtype).float() * factor[:, None]
        else:
            x = cache[at, :, j % page].float()
        return x.transpose(1, 2).contiguous()

    rows = lens[:, None] - T + torch.arange(T, device="cuda")
    i = rows[:, :, None]
    seen = (j <= i) & (pages >= 0)[:, None]
    if s["window"]:
        seen &= j > i - s["window"]
    if s["bounds"] is not None:
        lts, lte, uts, ute = (x[:, None] for x in s["bounds"])
        seen &= ~(((lts <= i) & (i < lte)) | ((uts <= i) & (i < ute)))
    scores = q.float().reshape(B, Hk, H // Hk * T, d) @ cached(s["k_cache"], s["k_scale"]).transpose(2, 3)
    scores = (scores * scale).view(B, Hk, H // Hk, T, -1).masked_fill(~seen[:, None, None], -math.inf)
    top = scores.amax(-1, keepdim=True)
    weights = (scores - torch.where(top == -math.inf, 0.0, top)).exp()
    total = weights.sum(-1, keepdim=True)
    lse = (top + total.log()).view(B, H, T)
    out = weights.view(B, Hk, H // Hk * T, -1) @ cached(s["v_cache"], s["v_scale"])
    out = out.view(B, H, T, d) / torch.where(total == 0, 1.0, total).view(B, H, T, 1)
    return out.to(q.dtype), lse


def _plain_fork(s):
    parents, new, page = s["parents"].long(), s["new_pages"], s["page"]
    lens = s["lens"][parents]
    rows = s["table"][parents]
    last = (lens // page)[:, None]
    col = torch.arange(rows.shape[1], device="cuda")
    copied = (new >= 0) & (lens % page != 0)
    table = torch.where((new >= 0)[:, None] & (col >= last), torch.where((col == last) & copied[:, None], new[:, None], -1), rows)
    source = rows.gather(1, last.long().clamp(max=rows.shape[1] - 1))[:, 0]
    to, source = new[copied].long(), source[copied].long()
    for pool in s["pools"]:
        raw = pool.view(torch.uint8) if pool.element_size() == 1 else pool
        raw[to] = raw[source]
    return table, lens, s["pools"]


def _plain_reclaim(s):
    table, total = s["table"], s["num_pages"]
    number = torch.arange(total, device="cuda")
    used = torch.zeros(total, dtype=torch.bool, device="cuda")
    used[table[table >= 0].long()] = True
    count = used.sum()
    free = torch.full((total,), -1, dtype=torch.int32, device="cuda")
    unused = number[~used]
    free[:unused.numel()] = unused.int()
    to, source = number[~used & (number < count)], number[used & (number >= count)]
    place = number.int()
    place[source] = to.int()
    for pool in s["pools"]:
        raw = pool.view(torch.uint8) if pool.element_size() == 1 else pool
        raw[to] = raw[source]
    return free, (total - count).int().view(1), torch.where(table >= 0, place[table.clamp(min=0).long()], table), count.int().view(1), s["pools"]


# --- the definitions in 64 bits: pairs as complex numbers, caches and tables sequence by sequence
def _turned(x, turn, interleaved):
    half = turn.shape[-1]
    x = x.double()
    head = x[..., :2 * half].unflatten(-1, (half, 2) if interleaved else (2, half))
    pair = torch.view_as_real(torch.view_as_complex((head if interleaved else head.transpose(-1, -2)).contiguous()) * turn)
    return torch.cat(((pair if interleaved else pair.transpose(-1, -2)).flatten(-2), x[..., 2 * half:]), -1)


def exact(case, seed):
    s = prepare(case, seed)
    kind = s["kind"]
    if kind == "rope":
        positions = s["positions"] if s["positions"] is not None else torch.arange(case["N"], device="cuda")[None]
        turn = s["amp"] * torch.exp(1j * (positions[:, None, :, None].double() * s["freqs"]))
        return tuple(_turned(s[n], turn if n in "qk" else turn.conj(), s["interleaved"]) for n in ("q", "k", "dq", "dk"))
    if kind == "append":
        turn = s["amp"] * torch.exp(1j * (s["positions"][:, None, None].double() * s["freqs"]))
        q, k, v = _turned(s["q"], turn, s["interleaved"]), _turned(s["k"], turn, s["interleaved"]), s["v"].double()
        caches = []
        seqs, at, table = s["seqs"].tolist(), s["positions"].tolist(), s["table"].tolist()
        place = [(n, table[b][p // s["page"]], p % s["page"]) for n, (b, p) in enumerate(zip(seqs, at)) if b >= 0]
        token, page, slot = (torch.tensor(x, device="cuda") for x in zip(*place))
        for x, cache, scale in ((k, s["k_cache"], s["k_scale"]), (v, s["v_cache"], s["v_scale"])):
            if scale is not None:
                x = (x / scale.double()[:, None]).clamp(-448, 448)
            caches.append(cache.double())
            caches[-1].transpose(1, 2)[page, slot] = x[token]
        return q, *caches
    if kind == "decode":
        B, H, T, d = s["q"].shape
        Hk, page = s["k_cache"].shape[1], s["page"]
        out = torch.zeros((B, H, T, d), dtype=torch.float64, device="cuda")
        lse = torch.full((B, H, T), -math.inf, dtype=torch.float64, device="cuda")
        for b, L in enumerate(s["lens"].tolist()):
            if L == 0:
                continue
            pages = s["table"][b, :-(-L // page)].long()
            keys, values = ((c.view(torch.uint8)[pages].view(c.dtype) if c.element_size() == 1 else c[pages]).double().transpose(1, 2)
                            .reshape(-1, Hk, d)[:L] for c in (s["k_cache"], s["v_cache"]))
            for t in range(T):
                i = L - T + t
                j = torch.arange(L, device="cuda")
                hidden = (j > i) | ((i - j >= s["window"]) if s["window"] else (j > L))
                if s["bounds"] is not None:
                    lts, lte, uts, ute = (x[b, :L] for x in s["bounds"])
                    hidden |= ((lts <= i) & (i < lte)) | ((uts <= i) & (i < ute))
                seen = j[~hidden]
                if not seen.numel():
                    continue
                for h in range(Hk):
                    group = slice(h * (H // Hk), (h + 1) * (H // Hk))
                    score = s["q"][b, group, t].double() @ keys[seen, h].T * s["scale"]
                    if s["k_scale"] is not None:
                        score = score * s["k_scale"][h].double()
                    lse[b, group, t] = torch.logsumexp(score, -1)
                    weight = torch.exp(score - lse[b, group, t][:, None])
                    out[b, group, t] = weight @ values[seen, h] * (1.0 if s["v_scale"] is None else s["v_scale"][h].double())
        return out, lse
    pools = [p.clone() for p in s["pools"]]
    table = s["table"].cpu().numpy()
    if kind == "fork":
        lens, parents, new = (s[n].cpu().numpy() for n in ("lens", "parents", "new_pages"))
        rows, moves = table[parents].copy(), []
        for r, (p, page) in enumerate(zip(parents, new)):
            if page >= 0:
                full, rest = divmod(int(lens[p]), s["page"])
                rows[r, full:] = -1
                if rest:
                    rows[r, full] = page
                    moves.append((int(table[p, full]), int(page)))
        result = [torch.from_numpy(rows), torch.from_numpy(lens[parents])]
    else:
        total = s["num_pages"]
        used = sorted(set(table[table >= 0].tolist()))
        unused = sorted(set(range(total)) - set(used))
        moves = list(zip([p for p in used if p >= len(used)], [p for p in unused if p < len(used)]))
        place = dict(moves)
        result = [torch.tensor(unused + [-1] * len(used), dtype=torch.int32), torch.tensor([len(unused)], dtype=torch.int32),
                  torch.from_numpy(np.vectorize(lambda p: place.get(p, p), otypes=[np.int32])(table)), torch.tensor([len(used)], dtype=torch.int32)]
    for pool, old in zip(pools, s["pools"]):
        for source, to in moves:
            pool[to].copy_(old[source])
    return *result, pools
