"""Performance cases of the operators that weigh a cache's keys and drop the light ones, and of those that verify a tree of
drafted tokens over the cache.

A case is one pass of what a serving program has them do.  `own` selects the library's entry points; without it the same
outputs come from elementary torch operations.  The cases run from a short prompt or a single sequence (nothing but latency) to
131072 keys and gigabytes of pages, over both head dimensions, the types and layouts that the entry points take, odd
lengths, empty sequences, padding and rows that see nothing.

Fields of a case, by kind:
  kind     "weights"  the attention weight that each key of a prompt gets from its query rows, all of them or the last ones
           "gather"   T new tokens of each sequence add theirs to the weights accumulated over the cache
           "evict"    sequences longer than `keep` keep their first, their last and their heaviest tokens, in new pages
           "tree"     T drafted tokens of each sequence, each with a parent, attend to the cache and to their ancestors
           "accept"   the drafted tokens of one path each are moved to consecutive places, in all layers
  B, H, Hk, N, T, d, page   sequences, query and K/V heads, (longest) length, new tokens, head dimension, tokens to a page
  type, cache               element types; an e4m3 cache has a scale for each K/V head
  packed                    tensors stored [B,N,H,d] and caches [pages,page,Hk,d], passed as strided views
  mask                      of a prompt: "causal", "docs", "encoder" (documents both ways, padding behind them), "window", "answers"
                            over a cache: "none", "window", "answers"
  rows                      query rows of a prompt that count, from its end; 0: all
  shared                    one selection for all heads of a sequence instead of one for each
  len_seed                  draws lengths, documents, trees and paths, which belong to the case (the tensors to the seed)
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

_TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "e4m3": torch.float8_e4m3fn}
_SIZE = {"bf16": 2, "f16": 2, "e4m3": 1}


def _weights(name, B, H, Hk, N, d, mask, rows=0, packed=False, len_seed=5):
    return {"name": name, "kind": "weights", "B": B, "H": H, "Hk": Hk, "N": N, "d": d, "mask": mask, "rows": rows, "packed": packed,
            "type": "bf16", "len_seed": len_seed}


def _gather(name, B, H, Hk, N, T, d, page, type, cache, mask="none", decay=1.0, packed=False, ragged=False, len_seed=5):
    return {"name": name, "kind": "gather", "B": B, "H": H, "Hk": Hk, "N": N, "T": T, "d": d, "page": page, "type": type,
            "cache": cache, "mask": mask, "decay": decay, "packed": packed, "ragged": ragged, "len_seed": len_seed}


def _evict(name, B, Hk, N, keep, first, recent, d, page, cache, shared=False, packed=False, ragged=False, len_seed=5):
    return {"name": name, "kind": "evict", "B": B, "Hk": Hk, "N": N, "keep": keep, "first": first, "recent": recent, "d": d, "page": page,
            "cache": cache, "shared": shared, "packed": packed, "ragged": ragged, "len_seed": len_seed}


def _tree(name, B, H, Hk, N, T, d, page, type, cache, mask="none", packed=False, ragged=False, len_seed=5):
    return {"name": name, "kind": "tree", "B": B, "H": H, "Hk": Hk, "N": N, "T": T, "d": d, "page": page, "type": type, "cache": cache,
            "mask": mask, "packed": packed, "ragged": ragged, "len_seed": len_seed}


def _accept(name, B, Hk, N, T, d, page, cache, pools, packed=False, len_seed=5):
    return {"name": name, "kind": "accept", "B": B, "Hk": Hk, "N": N, "T": T, "d": d, "page": page, "cache": cache, "pools": pools,
            "packed": packed, "ragged": True, "len_seed": len_seed}


def listed():
    return [
        # the smallest prompt: a few hundred tokens of two documents
        _weights("weights_docs_500", 1, 4, 2, 500, 64, "docs"),
        # a long prompt of a question with three answers, grouped heads, projections stored [B,N,H,d]: every row counts
        _weights("weights_answers_16384", 1, 32, 8, 16384, 128, "answers", packed=True),
        # the last rows of a very long prompt decide which of its keys are worth keeping
        _weights("weights_last_131072", 1, 32, 8, 131072, 128, "causal", rows=64),
        # one decoding step of 64 sequences of very different lengths, an empty one and one of a single token among them
        _gather("gather_ragged_8192", 64, 32, 8, 8192, 1, 128, 64, "bf16", "bf16", ragged=True),
        # the last 32 tokens of four prompts of questions with answers, 8-bit cache stored [pages,page,Hk,d], older weights fade
        _gather("gather_answers_e4m3", 4, 32, 4, 20000, 32, 64, 16, "f16", "e4m3", "answers", 0.9, packed=True, ragged=True),
        # 48 sequences of up to 6000 tokens go back to 2048 each, every head to tokens of its own
        _evict("evict_heads_6000", 48, 8, 6000, 2048, 4, 256, 128, 64, "bf16", ragged=True),
        # one long prompt in 8 bits goes back to an eighth, the same tokens in all heads
        _evict("evict_long_131072", 1, 8, 131072, 16384, 16, 1000, 128, 16, "e4m3", shared=True, packed=True),
        # the smallest tree: seven drafted tokens of one short sequence
        _tree("tree_400", 1, 8, 8, 400, 7, 64, 16, "bf16", "bf16"),
        # 16 ragged sequences verify trees of 63 tokens each
        _tree("tree_ragged_8192", 16, 32, 8, 8192, 63, 128, 64, "bf16", "bf16", ragged=True),
        # trees of 26 tokens over long windows of 8-bit caches stored [pages,page,Hk,d]
        _tree("tree_window_e4m3", 8, 16, 2, 30000, 26, 128, 32, "f16", "e4m3", "window", packed=True, ragged=True),
        # what eight sequences accept, one layer
        _accept("accept_8", 8, 8, 300, 20, 128, 16, "bf16", 2),
        # what 128 sequences accept, twelve layers
        _accept("accept_layers", 128, 8, 256, 63, 128, 64, "bf16", 24),
    ]


_MOST_BYTES, _MOST_FLOPS, _MOST_HELD = 3.7e8, 6e11, 9e9   # no drawn case moves or computes more than the largest listed one


def draw(rng):
    def spread(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    while True:
        kind = rng.choice(("weights", "weights", "gather", "gather", "evict", "evict", "tree", "tree", "accept"))
        d = rng.choice((64, 128, 128))
        Hk = rng.choice((1, 2, 4, 8, 8))
        H = Hk * rng.choice((1, 2, 4, 5, 8))
        seed = rng.randint(0, 1 << 30)
        page = rng.choice((16, 32, 64, 128, 256))
        type = rng.choice(("bf16", "bf16", "f16"))
        cache = rng.choice((type, type, "e4m3"))
        packed, ragged = rng.random() < 0.4, rng.random() < 0.7
        if kind == "weights":
            N = spread(100, 32768)
            rows = rng.choice((0, 0, 0, 32, 64, 200))
            case = _weights("", rng.choice((1, 1, 2, 4)), H, Hk, N, d, rng.choice(("causal", "docs", "encoder", "window", "answers")),
                            rows if rows < N else 0, packed, seed)
        elif kind == "gather":
            case = _gather("", spread(1, 96), H, Hk, spread(64, 65536), rng.choice((1, 1, 1, 2, 5, 16, 32)), d, page, type, cache,
                           rng.choice(("none", "none", "window", "answers")), rng.choice((1.0, 1.0, 0.75)), packed, ragged, seed)
        elif kind == "evict":
            N = spread(64, 65536)
            keep = max(16, int(N * rng.uniform(0.1, 0.9)))
            first = rng.choice((0, 1, 4))
            case = _evict("", spread(1, 64), Hk, N, keep, first, rng.randint(0, (keep - first) // 2), d, page, cache, rng.random() < 0.3,
                          packed, ragged, seed)
        elif kind == "tree":
            case = _tree("", spread(1, 48), H, Hk, spread(100, 32768), rng.choice((2, 5, 9, 16, 26, 40, 64)), d, page, type, cache,
                         rng.choice(("none", "none", "window", "answers")), packed, ragged, seed)
        else:
            case = _accept("", spread(1, 128), Hk, spread(80, 1024), rng.choice((5, 12, 26, 63)), d, page, cache, rng.choice((2, 4, 12)),
                           packed, seed)
        del case["name"]
        cost = work(case)
        if cost["bytes"] <= _MOST_BYTES and cost["flops"] <= _MOST_FLOPS and _held(case) <= _MOST_HELD:
            return case


# --- what belongs to a case: lengths, masks, trees, paths
_WINDOW = 1024


def _lengths(case):
    """Tokens of each sequence, the new ones among them; the longest has N.  A ragged batch has an empty and a one-token sequence in it."""
    B, N = case["B"], case["N"]
    rng = np.random.default_rng([case["len_seed"], 1])
    if not case["ragged"]:
        return np.full(B, N, np.int64)
    lens = np.exp(rng.uniform(math.log(max(1, N // 16)), math.log(N + 1), size=B)).astype(np.int64).clip(1, N)
    lens[0] = N
    if B >= 8:
        lens[3], lens[5] = 0, 1
    return lens


def _ends(case, L, rng):
    """Ends of the documents of a prompt."""
    cuts = np.sort(rng.integers(1, L, size=max(1, min(7, L // 200))))
    return np.append(np.unique(cuts), L)


def _prompt_bounds(case):
    """LTS, LTE, UTS, UTE [4, B, N] of a prompt's mask."""
    B, N = case["B"], case["N"]
    rng = np.random.default_rng([case["len_seed"], 2])
    at = np.arange(N)
    out = np.zeros((4, B, N), np.int64)
    for b in range(B):
        lts, lte, uts, ute = np.full(N, N), np.full(N, N), np.zeros(N, np.int64), at.copy()
        if case["mask"] == "window":
            lts = np.minimum(at + _WINDOW, N)
        elif case["mask"] == "docs":
            ends = _ends(case, N, rng)
            lts = ends[np.searchsorted(ends, at, side="right")]
        elif case["mask"] == "encoder":
            L = max(2, N - N // 9)               # documents both ways, and padding: its keys and rows see nothing of each other
            ends = np.append(_ends(case, L, rng), N)
            doc = np.searchsorted(ends, at, side="right")
            lts, ute = ends[doc], np.append(0, ends)[doc]
            lts[L:], ute[L:] = 0, N
        elif case["mask"] == "answers":
            ends = _answer_ends(N)
            for lo, hi in zip(ends[:-1], ends[1:]):
                lts[lo:hi] = hi
        out[:, b] = lts, lte, uts, ute
    return out


def _answer_ends(L):
    """A question (two fifths) and three answers."""
    question = L * 2 // 5
    return question + (L - question) * np.arange(4) // 3


def _cache_bounds(case):
    """LTS [B, N] of questions with three answers that do not see each other; the new tokens go on with the third."""
    lts = np.full((case["B"], case["N"]), case["N"], np.int64)
    for row, L in enumerate(_lengths(case)):
        ends = _answer_ends(int(L))
        lts[row, ends[0]:ends[1]] = ends[1]
        lts[row, ends[1]:ends[2]] = ends[2]
    return lts


def _visible(case):
    """Keys that at least one of a sequence's new tokens sees, per sequence."""
    lens, T = _lengths(case), case["T"]
    if case["mask"] == "window":
        return np.minimum(lens, _WINDOW + T - 1)
    if case["mask"] == "answers":
        question = lens * 2 // 5
        second = question + (lens - question) * 2 // 3
        return np.minimum(lens, question + lens - second + T - 1)
    return lens


def _seen_pairs(case):
    """Pairs (row, key) of a prompt that count, of one head."""
    bounds, N = _prompt_bounds(case), case["N"]
    first = N - case["rows"] if case["rows"] else 0
    lts, lte, uts, ute = bounds
    hidden = [np.clip(hi, first, N) - np.clip(lo, first, N) for lo, hi in ((lts, lte), (uts, ute))]
    both = np.minimum(np.clip(lte, first, N), np.clip(ute, first, N)) - np.maximum(np.clip(lts, first, N), np.clip(uts, first, N))
    union = sum(np.maximum(x, 0) for x in hidden) - np.maximum(both, 0)
    return int((N - first - union).sum())


def _parents(case):
    """Parent of each drafted token [B, T], -1: it follows the sequence itself."""
    rng = np.random.default_rng([case["len_seed"], 3])
    B, T = case["B"], case["T"]
    at = np.arange(T)
    reach = rng.integers(1, 13, size=(B, T))           # a parent is one of the tokens shortly before
    parents = at - reach
    return np.where((at < 4) | (parents < 0), np.where(rng.random((B, T)) < 0.5, -1, at - 1), parents)


def _paths(case):
    """Accepted tokens [B, P], ascending, -1 behind them.  A pass can be made again on the same pages: what is moved comes from behind all
    places that are written."""
    rng = np.random.default_rng([case["len_seed"], 4])
    B, T = case["B"], case["T"]
    P = min(T, 8)
    paths = np.full((B, P), -1, np.int64)
    for b in range(B):
        m = int(rng.integers(0, P + 1))
        stay = int(rng.integers(0, m + 1))             # a first part may be where it belongs
        paths[b, :stay] = np.arange(stay)
        moved = min(m - stay, T - m)
        paths[b, stay:stay + moved] = np.sort(rng.choice(np.arange(m, T), size=moved, replace=False))
    return paths


def _new_tokens_of(case):
    """Sequences that hold drafted tokens: the others are too short to."""
    return _lengths(case) >= case["T"]


def _token_bytes(case):
    return case["Hk"] * case["d"] * _SIZE[case["cache"]]


def _held(case):
    """Bytes of a state and of what the plain form makes of it."""
    if case["kind"] == "weights":
        return 4 * case["B"] * case["N"] * (case["H"] + case["Hk"]) * case["d"]
    tokens = int((_lengths(case) + case["page"]).sum())
    if case["kind"] == "evict":
        tokens += case["B"] * (case["keep"] + case["page"])
    plain = 0
    if case["kind"] in ("gather", "tree"):
        plain = 4 * case["B"] * case["N"] * (4 * case["Hk"] * case["d"] + 3 * case["H"] * case["T"])
    return case.get("pools", 2) * tokens * _token_bytes(case) + plain


def work(case):
    """Each input read once and each output written once."""
    kind, B, Hk, d = case["kind"], case["B"], case["Hk"], case["d"]
    if kind == "weights":
        H, N, rows = case["H"], case["N"], case["rows"] or case["N"]
        return {"bytes": B * (2 * d * (H * rows + Hk * N) + 4 * H * rows + 16 * N + 4 * Hk * N), "flops": 2 * d * case["H"] * _seen_pairs(case)}
    lens = _lengths(case)
    table = 4 * int((-(-lens // case["page"])).sum()) + 4 * B
    if kind in ("gather", "tree"):
        H, T = case["H"], case["T"]
        seen = int(_visible(case).sum())
        bounds = 16 * int(lens.sum()) if case["mask"] == "answers" else 0
        rows = B * T * H * d * _SIZE[case["type"]]
        if kind == "gather":
            return {"bytes": seen * _token_bytes(case) + rows + 4 * B * T * H + 8 * Hk * int(lens.sum()) + table + bounds,
                    "flops": 2 * H * T * d * seen}
        return {"bytes": 2 * seen * _token_bytes(case) + 2 * rows + 4 * B * T * H + 4 * B * T + table + bounds, "flops": 4 * H * T * d * seen}
    if kind == "evict":
        long = lens > case["keep"]
        heads = 1 if case["shared"] else Hk
        kept = int(np.minimum(lens, case["keep"]).sum())
        return {"bytes": 4 * int(long.sum()) * case["keep"] * _token_bytes(case) + heads * (4 * int(lens.sum()) + 4 * B * (case["N"] + case["keep"]))
                + 2 * table, "flops": kept}
    paths = _paths(case)[_new_tokens_of(case)]
    moved = int((paths > np.arange(paths.shape[1])).sum())
    return {"bytes": 2 * case["pools"] * moved * _token_bytes(case) + 4 * paths.size + 8 * B, "flops": 0}


# --- inputs
def _pool(case, pages, gen):
    """Pages of one layer's keys or values, indexed [page, head, token, d]."""
    shape = (pages, case["page"], case["Hk"], case["d"]) if case["packed"] else (pages, case["Hk"], case["page"], case["d"])
    x = torch.randn(shape, device="cuda", dtype=torch.bfloat16, generator=gen).to(_TYPES[case["cache"]])
    return x.transpose(1, 2) if case["packed"] else x


def _tables(counts, columns, gen, spare):
    """A page table with counts[b] pages of sequence b in random order, -1 behind them, the pages left over, and the number of pages."""
    counts = torch.from_numpy(counts).cuda()
    total = int(counts.sum())
    order = torch.randperm(total + spare, device="cuda", generator=gen).to(torch.int32)
    col = torch.arange(columns, device="cuda")
    at = (counts.cumsum(0) - counts)[:, None] + col
    return torch.where(col < counts[:, None], order[at.clamp(max=max(total - 1, 0))], -1), order[total:], total + spare


def _device(x):
    return torch.from_numpy(np.ascontiguousarray(x).astype(np.int32)).cuda()


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    kind = case["kind"]
    state = {"kind": kind, "scale": 1.0 / math.sqrt(case["d"])}

    def normal(*shape):
        return torch.randn(shape, device="cuda", generator=gen).to(_TYPES[case["type"]])

    if kind == "weights":
        B, N, d = case["B"], case["N"], case["d"]
        for name, heads in (("q", case["H"]), ("k", case["Hk"])):
            state[name] = normal(B, N, heads, d).transpose(1, 2) if case["packed"] else normal(B, heads, N, d)
        state["bounds"] = tuple(_device(x) for x in _prompt_bounds(case))
        state["first_row"] = N - case["rows"] if case["rows"] else 0
        state["lse"] = _prompt_lse(state)              # the attention call's second output
        state["scratch"] = torch.zeros(64 << 20, device="cuda", dtype=torch.uint8)   # kept by a serving program, as below
        return state

    lens, page = _lengths(case), case["page"]
    spare = case["B"] * -(-case["keep"] // page) if kind == "evict" else 3
    table, left, total = _tables(-(-lens // page), -(-case["N"] // page), gen, spare)
    state |= {"table": table, "lens": _device(lens), "page": page}
    if kind == "accept":
        return state | {"T": case["T"], "path": _device(_paths(case)), "pools": [_pool(case, total, gen) for _ in range(case["pools"])]}
    state |= {"k_cache": _pool(case, total, gen), "v_cache": _pool(case, total, gen), "max_len": case["N"]}
    state["k_scale"], state["v_scale"] = None, None
    if case["cache"] == "e4m3":
        state["k_scale"], state["v_scale"] = (torch.rand(case["Hk"], device="cuda", generator=gen) * 0.5 + 0.75 for _ in range(2))
    state["scratch"] = torch.zeros(128 << 20, device="cuda", dtype=torch.uint8)
    if kind == "evict":
        heads = 1 if case["shared"] else case["Hk"]
        # sums of softmax weights: many light keys, a few heavy ones, and some that were never looked at
        weights = torch.randn((case["B"], heads, case["N"]), device="cuda", generator=gen).mul(2.0).exp()
        weights *= torch.rand(weights.shape, device="cuda", generator=gen) > 0.1
        return state | {"weights": weights, "keep": case["keep"], "first": case["first"], "recent": case["recent"],
                        "new_table": left[:spare].view(case["B"], -1).contiguous()}
    B, H, T, d = case["B"], case["H"], case["T"], case["d"]
    state["q"] = normal(B, T, H, d).transpose(1, 2) if case["packed"] else normal(B, H, T, d)
    state["window"] = _WINDOW if case["mask"] == "window" else 0
    state["bounds"] = None
    if case["mask"] == "answers":
        lts = _device(_cache_bounds(case))
        state["bounds"] = (lts, torch.full_like(lts, case["N"]), torch.zeros_like(lts), torch.zeros_like(lts))
    if kind == "tree":
        return state | {"parents": _device(_parents(case))}
    state["lse"] = _attend(state, _cache_scores(state, *_causal(state)))[1]
    state["decay"] = case["decay"]
    state["weights"] = torch.rand((B, case["Hk"], case["N"]), device="cuda", generator=gen)
    state["out"] = torch.zeros_like(state["weights"])
    return state


# --- one pass
def run(state):
    if own:
        return {"weights": _own_weights, "gather": _own_gather, "evict": _own_evict, "tree": _own_tree, "accept": _own_accept}[state["kind"]](state)
    return {"weights": _plain_weights, "gather": _plain_gather, "evict": _plain_evict, "tree": _plain_tree,
            "accept": _plain_accept}[state["kind"]](state)


def _own_weights(s):
    import paper_2410_01359_amd as fm
    return fm.flashmask_weights(s["q"], s["k"], s["lse"], *s["bounds"], s["scale"], first_row=s["first_row"], workspace=s["scratch"])


def _own_gather(s):
    import paper_2410_01359_amd as fm
    return fm.flashmask_cache_weights(s["q"], s["k_cache"], s["v_cache"], s["table"], s["lens"], s["lse"], s["scale"], s["weights"], out=s["out"],
                                      decay=s["decay"], bounds=s["bounds"], window=s["window"], k_scale=s["k_scale"], v_scale=s["v_scale"])


def _own_evict(s):
    import paper_2410_01359_amd as fm
    table, lens, weights, kept = fm.flashmask_cache_evict(s["k_cache"], s["v_cache"], s["table"], s["lens"], s["weights"], s["new_table"], s["keep"],
                                                          first=s["first"], recent=s["recent"], k_scale=s["k_scale"], v_scale=s["v_scale"],
                                                          workspace=s["scratch"])
    return table, lens, weights, kept, s["k_cache"], s["v_cache"]


def _own_tree(s):
    import paper_2410_01359_amd as fm
    return fm.flashmask_decode_tree(s["q"], s["k_cache"], s["v_cache"], s["table"], s["lens"], s["parents"], s["scale"], bounds=s["bounds"],
                                    window=s["window"], k_scale=s["k_scale"], v_scale=s["v_scale"], workspace=s["scratch"])


def _own_accept(s):
    import paper_2410_01359_amd as fm
    return fm.flashmask_cache_accept(s["pools"], s["table"], s["lens"], s["T"], s["path"]), s["pools"]


# scores of a prompt's rows in pieces of this many at most
_PIECE = 1 << 28


def _prompt_scores(s, first):
    """(b, query heads, K/V head, rows, masked scores [heads, rows, N] in 32 bits), piece by piece."""
    B, H, N, d = s["q"].shape
    group = H // s["k"].shape[1]
    i = torch.arange(first, N, device="cuda")
    for b in range(B):
        lts, lte, uts, ute = (x[b] for x in s["bounds"])
        for hk in range(s["k"].shape[1]):
            keys = s["k"][b, hk].float().T.contiguous()
            step = max(1, _PIECE // (group * N))
            for rows in i.split(step):
                r = rows[:, None]
                hidden = ((lts <= r) & (r < lte)) | ((uts <= r) & (r < ute))
                heads = slice(hk * group, (hk + 1) * group)
                scores = s["q"][b, heads][:, rows].float() @ keys
                yield b, heads, hk, rows, (scores * s["scale"]).masked_fill_(hidden, -math.inf)


def _prompt_lse(s):
    B, H, N, _ = s["q"].shape
    lse = torch.full((B, H, N), -math.inf, device="cuda")
    for b, heads, _, rows, scores in _prompt_scores(s, s["first_row"]):
        top = scores.amax(-1, keepdim=True)
        ref = torch.where(top == -math.inf, 0.0, top)
        lse[b, heads][:, rows] = (ref + scores.sub_(ref).exp_().sum(-1, keepdim=True).log())[..., 0]
    return lse


def _plain_weights(s):
    B, _, N, _ = s["q"].shape
    out = torch.zeros((B, s["k"].shape[1], N), device="cuda")
    for b, heads, hk, rows, scores in _prompt_scores(s, s["first_row"]):
        lse = s["lse"][b, heads][:, rows][..., None]
        out[b, hk] += scores.sub_(torch.where(lse == -math.inf, math.inf, lse)).exp_().sum((0, 1))
    return out


def _places(s):
    """Page and slot of every place up to the longest sequence's last."""
    j = torch.arange(s["max_len"], device="cuda")
    return j, s["table"][:, j // s["page"]], j % s["page"]


def _cached(s, cache, factor):
    """A cache in the order of places [B, Hk, keys, d], in 32 bits."""
    _, pages, slot = _places(s)
    at = pages.clamp(min=0).long()
    if cache.element_size() == 1:
        x = cache.view(torch.uint8)[at, :, slot].view(cache.dtype).float() * factor[:, None]
    else:
        x = cache[at, :, slot].float()
    return x.transpose(1, 2).contiguous()


def _causal(s):
    """Rows [B, T] of the new tokens, positions [B, 1, keys] and which keys the causal rule lets them see [B, T, keys]."""
    T = s["q"].shape[2]
    rows = s["lens"][:, None] - T + torch.arange(T, device="cuda")
    j = torch.arange(s["max_len"], device="cuda")
    return rows, j[None, None], j <= rows[:, :, None]


def _drafted(s):
    """The same for a tree of drafted tokens."""
    B, T = s["parents"].shape
    at = torch.arange(T, device="cuda")
    reach = ((s["parents"][:, :, None] == at) | (at[:, None] == at)).float()     # a token and its parent; then all ancestors
    for _ in range(max(1, T - 1).bit_length()):
        reach = ((reach @ reach) > 0).float()
    depth = reach.sum(-1).int() - 1
    start = s["lens"][:, None] - T
    j = torch.arange(s["max_len"], device="cuda")
    u = j - start
    inside = (u >= 0) & (u < T)
    u = u.clamp(0, T - 1).long()
    ancestor = reach.gather(2, u[:, None].expand(B, T, -1)) > 0
    seen = torch.where(inside[:, None], ancestor, (j < start)[:, None]) & (start + at >= 0)[:, :, None]
    return start + depth, torch.where(inside, start + depth.gather(1, u), j)[:, None], seen


def _cache_scores(s, rows, positions, seen):
    """Masked scores [B, Hk, group, T, keys]."""
    B, H, T, d = s["q"].shape
    Hk = s["k_cache"].shape[1]
    _, pages, _ = _places(s)
    i = rows[:, :, None]
    seen = seen & (pages >= 0)[:, None]
    if s["window"]:
        seen &= positions > i - s["window"]
    if s["bounds"] is not None:
        lts, lte, uts, ute = (x[:, None] for x in s["bounds"])
        seen &= ~(((lts <= i) & (i < lte)) | ((uts <= i) & (i < ute)))
    scores = s["q"].float().reshape(B, Hk, H // Hk * T, d) @ _cached(s, s["k_cache"], s["k_scale"]).transpose(2, 3).contiguous()
    return (scores * s["scale"]).view(B, Hk, H // Hk, T, -1).masked_fill_(~seen[:, None, None], -math.inf)


def _attend(s, scores):
    """Softmax numerators and logsumexp [B, H, T] of scores, which are overwritten, and the sums of the former."""
    B, H, T, _ = s["q"].shape
    top = scores.amax(-1, keepdim=True)
    weights = scores.sub_(torch.where(top == -math.inf, 0.0, top)).exp_()
    total = weights.sum(-1, keepdim=True)
    return weights, (top + total.log()).view(B, H, T), total


def _plain_gather(s):
    scores = _cache_scores(s, *_causal(s))
    B, Hk, group, T, _ = scores.shape
    lse = s["lse"].view(B, Hk, group, T, 1)
    sums = scores.sub_(torch.where(lse == -math.inf, math.inf, lse)).exp_().sum((2, 3))
    j, lens = torch.arange(s["max_len"], device="cuda"), s["lens"][:, None, None]
    old = torch.where(j < lens - T, s["weights"] * s["decay"], 0.0)
    s["out"].copy_(torch.where(j < lens, old + sums, s["out"]))
    return s["out"]


def _plain_tree(s):
    B, H, T, d = s["q"].shape
    weights, lse, total = _attend(s, _cache_scores(s, *_drafted(s)))
    Hk = weights.shape[1]
    out = weights.view(B, Hk, H // Hk * T, -1) @ _cached(s, s["v_cache"], s["v_scale"])
    out = out.view(B, H, T, d) / torch.where(total == 0, 1.0, total).view(B, H, T, 1)
    return out.to(s["q"].dtype), lse


def _plain_evict(s):
    weights, lens, table, page, keep = s["weights"], s["lens"], s["table"], s["page"], s["keep"]
    B, heads, N = weights.shape
    Hk = s["k_cache"].shape[1]
    j, L = torch.arange(N, device="cuda"), lens[:, None, None]
    always = (j < s["first"]) | (j >= L - s["recent"])
    rank = torch.where(j >= L, -math.inf, torch.where(always, math.inf, weights))
    chosen = rank.sort(dim=-1, descending=True, stable=True).indices[..., :keep]
    count = L.clamp(max=keep)
    slots = torch.arange(keep, device="cuda")
    kept = torch.where(slots < count, chosen, N).sort(dim=-1).values
    there = slots < count
    at = torch.where(there, kept, 0)
    new_weights = torch.zeros_like(weights)
    new_weights[..., :keep] = torch.where(there, weights.gather(-1, at), 0.0)
    long = (lens > keep).nonzero()[:, 0]
    source = at[long].expand(-1, Hk, -1)
    pages = table[long][:, None].expand(-1, Hk, -1).gather(2, source // page).long()
    to = s["new_table"][long][:, slots // page].long()
    head = torch.arange(Hk, device="cuda")[:, None]
    for cache in (s["k_cache"], s["v_cache"]):
        raw = cache.view(torch.uint8) if cache.element_size() == 1 else cache
        raw[to[:, None], head, slots % page] = raw[pages, head, source % page]
    new_table = table.clone()
    new_table[long] = -1
    new_table[long, :s["new_table"].shape[1]] = s["new_table"][long]
    return new_table, count.view(B).int(), new_weights, torch.where(there, kept, -1).int(), s["k_cache"], s["v_cache"]


def _plain_accept(s):
    lens, path, page, T = s["lens"], s["path"], s["page"], s["T"]
    start = lens - T
    good = (path >= 0) & (start >= 0)[:, None]
    place = torch.arange(path.shape[1], device="cuda")
    b, i = (good & (path > place)).nonzero(as_tuple=True)
    to, source = start[b] + i, start[b] + path[b, i]
    to_page, page_of = (s["table"][b, x // page].long() for x in (to, source))
    for pool in s["pools"]:
        raw = pool.view(torch.uint8) if pool.element_size() == 1 else pool
        raw[to_page, :, to % page] = raw[page_of, :, source % page]
    return torch.where(start >= 0, start + good.sum(1), lens).int(), s["pools"]


# --- the definitions in 64 bits: sequence by sequence and head by head
def _hidden(bounds, i, j):
    """Whether bounds hide keys j from rows i."""
    lts, lte, uts, ute = (x[j] for x in bounds)
    return ((lts <= i) & (i < lte)) | ((uts <= i) & (i < ute))


def _exact_weights(s):
    q, k, lse = s["q"], s["k"], s["lse"].double()
    B, H, N, _ = q.shape
    Hk, first = k.shape[1], s["first_row"]
    out = torch.zeros((B, Hk, N), dtype=torch.float64, device="cuda")
    j = torch.arange(N, device="cuda")
    for b in range(B):
        bounds = [x[b] for x in s["bounds"]]
        for lo in range(first, N, 2048):
            i = torch.arange(lo, min(N, lo + 2048), device="cuda")
            hidden = _hidden(bounds, i[:, None], j)
            for h in range(H):
                row = lse[b, h, i]
                logits = (q[b, h, i].double() @ k[b, h // (H // Hk)].double().T) * s["scale"] - row[:, None]
                weight = torch.exp(logits)
                weight[hidden | torch.isneginf(row)[:, None]] = 0
                out[b, h // (H // Hk)] += weight.sum(0)
    return out


def _sequence(s, b, L):
    """Keys and values [Hk, L, d] of a sequence, as stored."""
    pages = s["table"][b, :-(-L // s["page"])].long()
    return ((c.view(torch.uint8)[pages].view(c.dtype) if c.element_size() == 1 else c[pages]).double().transpose(0, 1).flatten(1, 2)[:, :L]
            for c in (s["k_cache"], s["v_cache"]))


def _exact_over_cache(s):
    q = s["q"].double()
    B, H, T, d = q.shape
    group = H // s["k_cache"].shape[1]
    tree = s["kind"] == "tree"
    parents = s["parents"].tolist() if tree else [range(-1, T - 1)] * B
    if tree:
        out = torch.zeros((B, H, T, d), dtype=torch.float64, device="cuda")
        lses = torch.full((B, H, T), -math.inf, dtype=torch.float64, device="cuda")
    else:
        out = s["out"].double()
    for b, L in enumerate(s["lens"].tolist()):
        if L == 0:
            continue
        start = L - T
        lines = []                          # each drafted token's ancestors, itself among them
        for t, p in enumerate(parents[b]):
            lines.append((lines[p] if p >= 0 else []) + [t])
        keys, values = _sequence(s, b, L)
        j = torch.arange(L, device="cuda")
        position = j.clone()
        for t, line in enumerate(lines):
            if start + t >= 0:
                position[start + t] = start + len(line) - 1
        if not tree:
            out[b, :, :L] = 0
            if start > 0:
                out[b, :, :start] = s["weights"][b, :, :start].double() * s["decay"]
        for t, line in enumerate(lines):
            if start + t < 0:
                continue
            i = start + len(line) - 1
            seen = j < start
            seen[[start + u for u in line if start + u >= 0]] = True
            if s["window"]:
                seen &= i - position < s["window"]
            if s["bounds"] is not None:
                seen &= ~_hidden([x[b] for x in s["bounds"]], i, j)
            seen = j[seen]
            if not seen.numel():
                continue
            score = torch.stack([keys[h // group][seen] @ q[b, h, t] for h in range(H)]) * s["scale"]
            if s["k_scale"] is not None:
                score *= s["k_scale"].double().repeat_interleave(group)[:, None]
            if not tree:
                weight = torch.exp(score - s["lse"][b, :, t].double()[:, None])
                out[b][:, seen] += weight.unflatten(0, (-1, group)).sum(1)
                continue
            lse = torch.logsumexp(score, -1)
            weight = torch.exp(score - lse[:, None])
            lses[b, :, t] = lse
            for h in range(H):
                out[b, h, t] = weight[h] @ values[h // group][seen] * (1.0 if s["v_scale"] is None else s["v_scale"][h // group].double())
    return (out, lses) if tree else out


def _exact_evict(s):
    page, keep = s["page"], s["keep"]
    weights, table, new_table, lens = (s[n].cpu().numpy() for n in ("weights", "table", "new_table", "lens"))
    B, heads, _ = weights.shape
    Hk = s["k_cache"].shape[1]
    kept, new_weights = np.full((B, heads, keep), -1, np.int32), np.zeros(weights.shape)
    rows, pools = table.copy(), [p.clone() for p in (s["k_cache"], s["v_cache"])]
    for b, L in enumerate(lens):
        for h in range(heads):
            chosen = np.arange(L)
            if L > keep:
                last = L - s["recent"]
                middle = np.arange(s["first"], last)
                heavy = middle[np.lexsort((middle, -weights[b, h, middle]))[:keep - s["first"] - s["recent"]]]
                chosen = np.concatenate((np.arange(s["first"]), np.sort(heavy), np.arange(last, L)))
            kept[b, h, :len(chosen)] = chosen
            new_weights[b, h, :len(chosen)] = weights[b, h, chosen]
        if L <= keep:
            continue
        rows[b] = -1
        rows[b, :new_table.shape[1]] = new_table[b]
        slot = np.arange(keep)
        to, to_slot = (torch.from_numpy(x).long().cuda() for x in (new_table[b, slot // page], slot % page))
        for h in range(Hk):
            at = kept[b, h if heads > 1 else 0]
            source, at_slot = (torch.from_numpy(x).long().cuda() for x in (table[b, at // page], at % page))
            for pool in pools:
                raw = pool.view(torch.uint8) if pool.element_size() == 1 else pool
                raw[to, h, to_slot] = raw[source, h, at_slot]
    return (torch.from_numpy(rows), torch.from_numpy(np.minimum(lens, keep)), torch.from_numpy(new_weights), torch.from_numpy(kept),
            *(p.double() for p in pools))


def _exact_accept(s):
    table, path, lens = (s[n].tolist() for n in ("table", "path", "lens"))
    page, T = s["page"], s["T"]
    moves, new_lens = [], []
    for b, L in enumerate(lens):
        if L < T:
            new_lens.append(L)
            continue
        line = [t for t in path[b] if t >= 0]
        new_lens.append(L - T + len(line))
        moves += [(b, L - T + t, L - T + i) for i, t in enumerate(line) if t != i]
    pools = [p.clone() for p in s["pools"]]
    if moves:
        source, slot, to, to_slot = (torch.tensor(x, device="cuda") for x in zip(*((table[b][x // page], x % page, table[b][y // page], y % page)
                                                                                    for b, x, y in moves)))
        for pool in pools:
            raw = pool.view(torch.uint8) if pool.element_size() == 1 else pool
            raw[to, :, to_slot] = raw[source, :, slot]
    return torch.tensor(new_lens), [p.float() for p in pools]


def exact(case, seed):
    s = prepare(case, seed)
    return {"weights": _exact_weights, "gather": _exact_over_cache, "tree": _exact_over_cache, "evict": _exact_evict,
            "accept": _exact_accept}[s["kind"]](s)
