"""Performance cases of the operators around a decoding step with several continuations: query/key norms
with the rotary append, log probabilities of tokens, forks of paged sequences.

A serving program that keeps several continuations of a request (best of n, beams) forks the requests' pages
(`page_fork`), per layer normalises, rotates and appends the new tokens (`prompt_norm_rope_append`, or
`tree_norm_rope_append` for a draft tree), and scores tokens from the hidden states (`lm_head_logprobs`) or from logits
that it has (`token_logprobs`): log probabilities of the tokens taken, entropies and the best alternatives.  `listed()`
holds fixed sizes, `draw()` further ones of the same ranges.  `plain` forms are elementary torch operations in 32 bits.
"""
from __future__ import annotations

import math
import random

import numpy as np
import torch

own = False

DEV = "cuda"
ROPE_BASE = 500000.0
EPS = 1e-6
MAX_LM_FLOPS = 4.4e12        # of one pass: the largest listed case (lm_score_4096)
MAX_BYTES = 2.2e9            # what a drawn case of another kind moves at most
MAX_CACHE = 1 << 30          # elements of a fork's K (and of its V)


def listed():
    return [
        # one decoded token for each of eight ragged requests, from fused QKV rows, 16-token pages, 32q/8kv
        {"name": "norm_decode_8", "kind": "norm", "dtype": "bf16", "hq": 32, "hkv": 8, "d": 128, "page": 16, "batch": 8,
         "new": 1, "ctx": 4096, "ragged": True, "mix": 1, "pad": 0},
        # a long prompt
        {"name": "norm_prompt_8192", "kind": "norm", "dtype": "bf16", "hq": 32, "hkv": 8, "d": 128, "page": 0, "batch": 1,
         "new": 8192, "ctx": 0, "ragged": False, "mix": 0, "pad": 0},
        # ragged prompts of a small model kept in fp32, padded to a captured size
        {"name": "norm_f32", "kind": "norm", "dtype": "f32", "hq": 16, "hkv": 8, "d": 64, "page": 32, "batch": 5, "new": 509,
         "ctx": 100, "ragged": True, "mix": 3, "pad": 19},
        # one draft tree through all layers of a model (its queries and keys at once)
        {"name": "tree_norm_32_layers", "kind": "tree", "dtype": "bf16", "hq": 32, "hkv": 8, "d": 128, "page": 0, "batch": 1,
         "nodes": 63, "layers": 32, "ctx": 8192, "ragged": False, "mix": 0},
        # eight ragged trees over pages, one layer
        {"name": "tree_norm_batch", "kind": "tree", "dtype": "bf16", "hq": 32, "hkv": 8, "d": 128, "page": 64, "batch": 8,
         "nodes": 64, "layers": 1, "ctx": 1000, "ragged": True, "mix": 2},
        # one decoded token
        {"name": "logprobs_1", "kind": "logprobs", "dtype": "bf16", "rows": 1, "vocab": 128256, "k": 8, "temperature": 1.0,
         "masked": 0.0},
        # a draft tree's nodes, under a grammar that allows a part of the vocabulary
        {"name": "logprobs_63", "kind": "logprobs", "dtype": "bf16", "rows": 63, "vocab": 128256, "k": 4, "temperature": 0.7,
         "masked": 0.9},
        # a chunk of a prompt's logits in fp32
        {"name": "logprobs_f32_1021", "kind": "logprobs", "dtype": "f32", "rows": 1021, "vocab": 32000, "k": 16,
         "temperature": 1.0, "masked": 0.0},
        # a decoding batch from its hidden states
        {"name": "lm_decode_63", "kind": "lm", "rows": 63, "vocab": 128256, "d": 4096, "k": 8, "temperature": 1.0},
        # the largest: the tokens of a prompt scored
        {"name": "lm_score_4096", "kind": "lm", "rows": 4096, "vocab": 128256, "d": 4096, "k": 4, "temperature": 1.0},
        # one prompt continued 64 times, 32 layers
        {"name": "fork_best_of_64", "kind": "fork", "dtype": "bf16", "hkv": 8, "d": 128, "layers": 32, "page": 16,
         "requests": 1, "beams": 1, "into": 64, "ctx": 2043, "tail": 0, "ended": 0.0, "mix": 1},
        # beams of 32 requests after a step, some requests finished
        {"name": "fork_beams_32x4", "kind": "fork", "dtype": "bf16", "hkv": 8, "d": 128, "layers": 8, "page": 16,
         "requests": 32, "beams": 4, "into": 4, "ctx": 900, "tail": 200, "ended": 0.1, "mix": 2},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["norm", "norm", "tree", "logprobs", "logprobs", "lm", "fork"])
    while True:
        if kind == "logprobs":
            c = {"kind": kind, "dtype": rng.choice(["bf16", "f32"]), "rows": _log(rng, 1, 4096),
                 "vocab": rng.choice([128256, 32000, _log(rng, 1000, 262144)]), "k": rng.choice([1, 2, 5, 8, 16]),
                 "temperature": rng.choice([1.0, 0.6, 1.3]), "masked": rng.choice([0.0, 0.0, 0.5, 0.99])}
        elif kind == "lm":
            c = {"kind": kind, "rows": _log(rng, 1, 8192), "vocab": rng.choice([128256, 32000, _log(rng, 1000, 200000)]),
                 "d": 64 * _log(rng, 8, 96), "k": rng.choice([1, 4, 8, 16]), "temperature": rng.choice([1.0, 0.7])}
            if work(c)["flops"] > MAX_LM_FLOPS:
                continue
            return c
        elif kind == "fork":
            c = {"kind": kind, "dtype": rng.choice(["bf16", "bf16", "f32"]), "hkv": rng.choice([1, 2, 8]),
                 "d": 128, "layers": _log(rng, 1, 32), "page": rng.choice([16, 32, 64, 128]),
                 "requests": _log(rng, 1, 128), "beams": rng.choice([1, 2, 4, 8]), "into": rng.choice([1, 2, 4, 8, 16]),
                 "ctx": _log(rng, 1, 8192), "tail": rng.choice([0, _log(rng, 1, 300)]), "ended": rng.choice([0.0, 0.1, 0.5]),
                 "mix": rng.randrange(1 << 20)}
            if _fork_pages(c) * c["page"] * c["hkv"] * c["d"] * c["layers"] > MAX_CACHE:
                continue
        else:
            c = {"kind": kind, "dtype": "bf16" if rng.random() < 0.8 else "f32", "page": rng.choice([0, 16, 32, 64, 128]),
                 "batch": 1 if rng.random() < 0.4 else _log(rng, 2, 64), "ctx": 0 if rng.random() < 0.3 else _log(rng, 1, 16384),
                 "ragged": rng.random() < 0.7, "mix": rng.randrange(1 << 20)}
            if c["dtype"] == "bf16":
                c["hq"], c["hkv"] = rng.choice([(32, 32), (32, 8), (64, 8), (16, 2), (28, 4), (40, 8)])
                c["d"] = 128
            else:
                c["hq"], c["hkv"] = rng.choice([(8, 8), (16, 16), (32, 8)])
                c["d"] = rng.choice([32, 64, 128])
            if kind == "norm":
                c["new"] = 1 if rng.random() < 0.2 else _log(rng, 2, 16384)
                c["pad"] = rng.choice([0, 0, rng.randrange(1, 200)])
            else:
                c["nodes"] = _log(rng, 1, 128)
                c["layers"] = rng.choice([1, 1, _log(rng, 2, 32)])
            ctx, new = _lengths(c)
            cells = (sum(ctx) + sum(new)) if c["page"] else len(new) * max(a + b for a, b in zip(ctx, new))
            if cells * c.get("layers", 1) * c["hkv"] * c["d"] > MAX_CACHE:
                continue
        if work(c)["bytes"] > MAX_BYTES:
            continue
        return c


def _lengths(case):
    """Contexts and numbers of new tokens (or tree nodes), host lists: a function of the case alone."""
    rng = random.Random(case["mix"])
    most = case["new"] if case["kind"] == "norm" else case["nodes"]
    ctx, new = [], []
    for b in range(case["batch"]):
        ragged = case["ragged"] and b > 0
        new.append(_log(rng, 1, most) if ragged else most)
        ctx.append(_log(rng, max(1, case["ctx"] // 4), case["ctx"]) if ragged and case["ctx"] else case["ctx"])
    return ctx, new


def _fork_plan(case):
    """A fork's source rows as page ids 0, 1, ..., the tokens in each, and the parents and lengths of the target."""
    rng = random.Random(case["mix"])
    P = case["page"]
    rows, tokens, parents, lens = [], [], [], []
    pages = 0
    for _ in range(case["requests"]):
        prefix = max(1, case["ctx"] - rng.randrange(0, max(1, case["ctx"] // 2)) if case["requests"] > 1 else case["ctx"])
        tail = 0 if case["tail"] == 0 else rng.randrange(1, case["tail"] + 1)
        first = len(rows)
        shared = prefix // P if case["beams"] > 1 else 0   # full pages that the beams of a request have in common
        common = list(range(pages, pages + shared))
        pages += shared
        for _ in range(case["beams"]):
            n = prefix + tail
            mine = -(-n // P) - shared
            rows.append(common + list(range(pages, pages + mine)))
            tokens.append(n)
            pages += mine
        ended = rng.random() < case["ended"]
        for _ in range(case["into"]):
            p = first + rng.randrange(case["beams"])
            parents.append(-1 if ended else p)
            lens.append(0 if ended else tokens[p])
    return rows, tokens, parents, lens, pages


def _fork_pages(case):
    rows, _, parents, _, pages = _fork_plan(case)
    return pages + len(parents) + 7


def _size(dtype):
    return 2 if dtype == "bf16" else 4


def _type(dtype):
    return torch.bfloat16 if dtype == "bf16" else torch.float32


def work(case):
    kind = case["kind"]
    if kind == "logprobs":
        n, v = case["rows"], case["vocab"]
        return {"bytes": n * v * _size(case["dtype"]) + n * (12 + 8 * case["k"]), "flops": 6 * n * v}
    if kind == "lm":
        n, v, d = case["rows"], case["vocab"], case["d"]
        return {"bytes": 2 * (n + v) * d + n * (12 + 8 * case["k"]), "flops": 2 * n * v * d}
    if kind == "fork":
        rows, _, parents, lens, pages = _fork_plan(case)
        P = case["page"]
        takers = {}
        for b, (p, n) in enumerate(zip(parents, lens)):
            if p >= 0 and n % P:
                takers.setdefault(rows[p][n // P], []).append(n % P)
        copied = sum(sum(x) - max(x) for x in takers.values())
        entries = sum(map(len, rows)) + sum(-(-n // P) for n in lens)
        moved = 2 * 2 * copied * case["layers"] * case["hkv"] * case["d"] * _size(case["dtype"])
        return {"bytes": moved + 4 * entries + 4 * (2 * len(rows) + 3 * len(parents)), "flops": 2 * entries}
    ctx, new = _lengths(case)
    N, L, d, hq, hkv = sum(new), case.get("layers", 1), case["d"], case["hq"], case["hkv"]
    return {"bytes": L * N * (2 * hq + 4 * hkv) * d * _size(case["dtype"]) + 8 * N, "flops": 7 * L * N * (hq + hkv) * d}


class State:
    pass


def prepare(case, seed):
    s = State()
    s.case = case
    g = torch.Generator(device=DEV).manual_seed(seed)
    host = np.random.default_rng(seed)
    s.status = torch.zeros(1, dtype=torch.int32, device=DEV)
    {"norm": _prepare_norm, "tree": _prepare_tree, "logprobs": _prepare_logprobs, "lm": _prepare_lm,
     "fork": _prepare_fork}[case["kind"]](s, case, g, host)
    return s


def _normal(g, shape, t):
    return torch.randn(shape, generator=g, device=DEV, dtype=torch.float32).to(t)


def _cache(s, case, host, g, ctx, new, layers, spare):
    """K and V that hold what they may, the block table (paged) and every sequence's rows."""
    i32 = dict(dtype=torch.int32, device=DEV)
    t, page, B, hkv, d = _type(case["dtype"]), case["page"], len(new), case["hkv"], case["d"]
    longest = max(c + n for c, n in zip(ctx, new))
    s.block_table = None
    if page:
        per = [-(-(c + n) // page) for c, n in zip(ctx, new)]
        num_pages = sum(per) + 3
        perm = host.permutation(num_pages).astype(np.int32)
        table = np.zeros((B, max(per)), np.int32)
        at = 0
        for b, n in enumerate(per):
            table[b, :n] = perm[at:at + n]
            at += n
        s.block_table = torch.tensor(table, **i32)
        shape = (layers, num_pages, page, hkv, d)
    else:
        shape = (layers, B, longest + spare, hkv, d)
    s.k, s.v = _normal(g, shape, t), _normal(g, shape, t)


def _rows(s, b, lo, hi):
    """Cache rows (of a layer) of sequence b's slots lo .. hi - 1."""
    p = torch.arange(lo, hi, device=DEV)
    if s.block_table is None:
        return b * s.k.shape[2] + p
    page = s.case["page"]
    return s.block_table[b].long()[p // page] * page + p % page


def _norm_weights(g, shape, t):
    return (1.0 + 0.2 * torch.randn(shape, generator=g, device=DEV, dtype=torch.float32)).to(t)


def _prepare_norm(s, case, g, host):
    i32 = dict(dtype=torch.int32, device=DEV)
    ctx, new = _lengths(case)
    s.ctx, s.new, s.off = ctx, new, [0] + [int(x) for x in np.cumsum(new)]
    t, hq, hkv, d, N = _type(case["dtype"]), case["hq"], case["hkv"], case["d"], s.off[-1] + case["pad"]
    s.N = N
    _cache(s, case, host, g, ctx, new, 1, 5)
    qkv = _normal(g, (N, (hq + 2 * hkv) * d), t)
    s.q = qkv[:, :hq * d].view(N, hq, d)
    s.kn = qkv[:, hq * d:(hq + hkv) * d].view(N, hkv, d)
    s.vn = qkv[:, (hq + hkv) * d:].view(N, hkv, d)
    s.wq, s.wk = _norm_weights(g, (d,), t), _norm_weights(g, (d,), t)
    s.q_out = torch.zeros((N, hq, d), dtype=t, device=DEV)
    s.token_offsets, s.ctx_lens = torch.tensor(s.off, **i32), torch.tensor(ctx, **i32)
    s.slots, s.positions = torch.full((N,), -1, **i32), torch.full((N,), -1, **i32)
    for b in range(len(new)):
        s.slots[s.off[b]:s.off[b + 1]] = _rows(s, b, ctx[b], ctx[b] + new[b]).to(torch.int32)
        s.positions[s.off[b]:s.off[b + 1]] = torch.arange(ctx[b], ctx[b] + new[b], **i32)
    if own:   # descriptions of the buffers above, which a program keeps
        from paper_2607_10661_gb300 import ptd
        s.cache = ptd.KVCache(s.k, s.v, hkv, d, case["page"], s.block_table)
        s.prompt = ptd.Prompt(s.token_offsets, s.ctx_lens, N, max(new), max(ctx))


def _prepare_tree(s, case, g, host):
    i32 = dict(dtype=torch.int32, device=DEV)
    ctx, new = _lengths(case)
    s.ctx, s.new, s.off = ctx, new, [0] + [int(x) for x in np.cumsum(new)]
    t, hq, hkv, d, N, L = _type(case["dtype"]), case["hq"], case["hkv"], case["d"], s.off[-1], case["layers"]
    s.N = N
    _cache(s, case, host, g, ctx, new, L, 5)
    s.q, s.kn, s.vn = _normal(g, (L, N, hq, d), t), _normal(g, (L, N, hkv, d), t), _normal(g, (L, N, hkv, d), t)
    s.wq, s.wk = _norm_weights(g, (L, d), t), _norm_weights(g, (L, d), t)
    s.q_out = torch.zeros_like(s.q)
    s.parents_host = []
    for n in new:   # a node's parent is one of the eight before it
        s.parents_host += [-1] + [int(host.integers(max(0, i - 8), i)) for i in range(1, n)]
    s.node_offsets, s.ctx_lens = torch.tensor(s.off, **i32), torch.tensor(ctx, **i32)
    s.parents = torch.tensor(s.parents_host, **i32)
    s.positions = torch.zeros(N, **i32)
    if own:
        from paper_2607_10661_gb300 import ptd
        s.cache = ptd.KVCache(s.k, s.v, hkv, d, case["page"], s.block_table)
        s.tree = ptd.Tree(s.node_offsets, s.parents, s.ctx_lens, max(new), max(ctx))


def _outputs(s, rows, k):
    s.logprob, s.entropy = torch.zeros(rows, device=DEV), torch.zeros(rows, device=DEV)
    s.top_idx = torch.zeros((rows, k), dtype=torch.int32, device=DEV)
    s.top_val = torch.zeros((rows, k), device=DEV)


def _prepare_logprobs(s, case, g, host):
    n, v = case["rows"], case["vocab"]
    x = 2.5 * torch.randn((n, v), generator=g, device=DEV)
    peak = torch.randint(0, v, (n,), generator=g, device=DEV)
    if case["masked"]:
        x.masked_fill_(torch.rand((n, v), generator=g, device=DEV) < case["masked"], -math.inf)
    x[torch.arange(n, device=DEV), peak] = 6.0 + 8.0 * torch.rand(n, generator=g, device=DEV)
    s.logits = x.to(_type(case["dtype"]))
    other = torch.randint(0, v, (n,), generator=g, device=DEV)   # half the tokens are unlikely ones, where the mask has them
    allowed = torch.isfinite(x[torch.arange(n, device=DEV), other]) & (torch.rand(n, generator=g, device=DEV) < 0.5)
    s.tokens = torch.where(allowed, other, peak).to(torch.int32)
    _outputs(s, n, case["k"])


def _prepare_lm(s, case, g, host):
    """Hidden states and weights in steps of 1/8 and about 1/2 / sqrt(d) (a power of two): their products' sums are
    whole numbers below 2^24 of one unit, so that the order of the alternatives does not hang on how they are summed."""
    n, v, d = case["rows"], case["vocab"], case["d"]
    unit = 2.0 ** -round(math.log2(math.sqrt(d)))
    grid = lambda shape: torch.randn(shape, generator=g, device=DEV).mul_(8.0).round_().mul_(0.125)
    s.hidden = grid((n, d)).to(torch.bfloat16)
    s.weight = grid((v, d)).mul_(4.0 * unit).to(torch.bfloat16)
    tokens = torch.randint(0, v, (n,), generator=g, device=DEV)
    s.tokens = tokens.to(torch.int32)
    _outputs(s, n, case["k"])
    if own:   # the scratch that a program keeps
        from paper_2607_10661_gb300 import ptd
        s.workspace = torch.empty(ptd.lm_head_logprobs_workspace_size(n, v, case["k"]), dtype=torch.uint8, device=DEV)


def _prepare_fork(s, case, g, host):
    i32 = dict(dtype=torch.int32, device=DEV)
    rows, tokens, parents, lens, pages = _fork_plan(case)
    t, P, L, hkv, d = _type(case["dtype"]), case["page"], case["layers"], case["hkv"], case["d"]
    num_pages = _fork_pages(case)
    perm = host.permutation(num_pages).astype(np.int32)
    width = max(max(map(len, rows)), -(-max(lens) // P)) + 2
    table = np.full((len(rows), width), -1, np.int32)
    for b, r in enumerate(rows):
        table[b, :len(r)] = perm[r]
    free = np.full(num_pages, -1, np.int32)
    free[:num_pages - pages] = perm[pages:]
    s.table, s.held = torch.tensor(table, **i32), torch.tensor([len(r) for r in rows], **i32)
    s.free, s.count = torch.tensor(free, **i32), torch.tensor([num_pages - pages], **i32)
    s.parents, s.lens = torch.tensor(parents, **i32), torch.tensor(lens, **i32)
    s.new_table, s.new_held = torch.full((len(parents), width), -1, **i32), torch.zeros(len(parents), **i32)
    s.new_free, s.new_count = torch.full((num_pages,), -1, **i32), torch.zeros(1, **i32)
    s.host = (table, [len(r) for r in rows], free, num_pages - pages, parents, lens)
    s.k, s.v = _normal(g, (L, num_pages, P, hkv, d), t), _normal(g, (L, num_pages, P, hkv, d), t)
    if own:
        from paper_2607_10661_gb300 import ptd
        s.cache = ptd.KVCache(s.k, s.v, hkv, d, P, s.table)
        s.source = ptd.PageSet(s.table, s.held, s.free, s.count)
        s.target = ptd.PageSet(s.new_table, s.new_held, s.new_free, s.new_count)
        s.workspace = torch.empty(ptd.page_fork_workspace_size(s.cache, s.source, s.target), dtype=torch.uint8, device=DEV)


def run(s):
    case, kind = s.case, s.case["kind"]
    if own:
        from paper_2607_10661_gb300 import ptd
        if kind == "norm":
            ptd.prompt_norm_rope_append(s.prompt, s.cache, 0, s.slots, s.positions, s.q, s.kn, s.vn, s.q_out, s.wq, s.wk, EPS,
                                        ROPE_BASE, s.status)
        elif kind == "tree":
            ptd.tree_norm_rope_append(s.tree, s.cache, 0, s.q, s.kn, s.vn, s.q_out, s.wq, s.wk, EPS, ROPE_BASE, s.status,
                                      s.positions)
        elif kind == "logprobs":
            ptd.token_logprobs(s.logits, s.tokens, s.logprob, s.entropy, s.top_idx, s.top_val, s.status, case["temperature"])
        elif kind == "lm":
            ptd.lm_head_logprobs(s.hidden, s.weight, s.tokens, s.logprob, s.entropy, s.top_idx, s.top_val, s.workspace, s.status,
                                 case["temperature"])
        else:
            ptd.page_fork(s.cache, s.source, s.target, s.parents, s.lens, s.workspace, s.status)
    else:
        {"norm": _plain_norm, "tree": _plain_tree, "logprobs": _plain_logprobs, "lm": _plain_lm, "fork": _plain_fork}[kind](s)
    if kind == "norm":
        return {"q": s.q_out, "k": s.k, "v": s.v}
    if kind == "tree":
        return {"q": s.q_out, "k": s.k, "v": s.v, "positions": s.positions}
    if kind == "fork":
        return {"k": s.k, "v": s.v, "block_table": s.new_table, "held": s.new_held, "free_pages": s.new_free,
                "free_count": s.new_count}
    return {"logprob": s.logprob, "entropy": s.entropy, "top_idx": s.top_idx, "top_val": s.top_val}


def _normed_turned(x, w, pos):
    """x [..., heads, D] over tokens at `pos`, w [D] or broadcastable: RMS norm of a head, then the rotation."""
    d = x.shape[-1]
    y = x.float()
    y = y * torch.rsqrt(y.square().mean(-1, keepdim=True) + EPS) * w.float()
    j = torch.arange(d // 2, device=DEV, dtype=torch.float64)
    angle = pos[:, None].double() * torch.pow(torch.tensor(ROPE_BASE, device=DEV, dtype=torch.float64), -2.0 * j / d)
    c, sn = angle.cos().float()[:, None, :], angle.sin().float()[:, None, :]
    a, b = y[..., :d // 2], y[..., d // 2:]
    return torch.cat([a * c - b * sn, a * sn + b * c], -1).to(x.dtype)


def _plain_norm(s):
    n = s.off[-1]   # the rows behind the last request stay as they were
    pos, rows = s.positions[:n], s.slots[:n].long()
    s.q_out[:n] = _normed_turned(s.q[:n], s.wq, pos)
    s.k.view(-1, *s.k.shape[3:])[rows] = _normed_turned(s.kn[:n], s.wk, pos)
    s.v.view(-1, *s.v.shape[3:])[rows] = s.vn[:n]


def _plain_tree(s):
    b = torch.repeat_interleave(torch.arange(len(s.new), device=DEV), s.node_offsets[1:].long() - s.node_offsets[:-1].long())
    start = s.node_offsets[:-1].long()[b]
    up = torch.where(s.parents >= 0, s.parents.long() + start, -1)
    depth, at = torch.zeros_like(up), up
    for _ in range(max(s.new)):   # ancestors, one level at a time
        there = at >= 0
        depth += there
        at = torch.where(there, up[at.clamp(min=0)], -1)
    ctx = s.ctx_lens.long()[b]
    s.positions.copy_(ctx + depth)
    slot = ctx + torch.arange(s.N, device=DEV) - start
    if s.block_table is None:
        rows = b * s.k.shape[2] + slot
    else:
        page = s.case["page"]
        rows = s.block_table.long()[b, slot // page] * page + slot % page
    L, hkv, d = s.k.shape[0], s.case["hkv"], s.case["d"]
    s.q_out.copy_(_normed_turned(s.q, s.wq[:, None, None, :], s.positions))
    s.k.view(L, -1, hkv, d)[:, rows] = _normed_turned(s.kn, s.wk[:, None, None, :], s.positions)
    s.v.view(L, -1, hkv, d)[:, rows] = s.vn


def _plain_row_logprobs(s, x, r0):
    """Outputs of rows r0 .. of 32-bit logits x."""
    n, v = x.shape
    k, out = s.case["k"], slice(r0, r0 + x.shape[0])
    z = x / s.case["temperature"]
    m = z.amax(-1, keepdim=True)
    e = (z - m).exp()
    total = e.sum(-1, keepdim=True)
    lse = m + total.log()
    s.logprob[out] = (z.gather(1, s.tokens[out].long()[:, None]) - lse)[:, 0]
    s.entropy[out] = total.log()[:, 0] - ((z - m).clamp(min=-1e4) * e).sum(-1) / total[:, 0]
    index, taken = torch.arange(v, device=DEV), torch.zeros_like(x, dtype=torch.bool)
    for j in range(k):   # the largest one left, the lowest index of equal ones
        best = x.masked_fill(taken, -math.inf).amax(-1, keepdim=True)
        at = torch.where((x == best) & ~taken, index, v).amin(-1, keepdim=True)
        taken.scatter_(1, at, True)
        s.top_idx[out, j] = at[:, 0].to(torch.int32)
        s.top_val[out, j] = (z.gather(1, at) - lse)[:, 0]


def _plain_logprobs(s):
    step = max(1, (1 << 28) // s.case["vocab"])
    for r0 in range(0, s.case["rows"], step):
        _plain_row_logprobs(s, s.logits[r0:r0 + step].float(), r0)


def _plain_lm(s):
    w = s.weight.float()
    step = max(1, (1 << 28) // s.case["vocab"])
    for r0 in range(0, s.case["rows"], step):
        _plain_row_logprobs(s, torch.matmul(s.hidden[r0:r0 + step].float(), w.t()), r0)


def _plain_fork(s):
    P, num_pages = s.case["page"], s.free.numel()
    B, width = s.table.shape
    none = 1 << 30
    column = torch.arange(width, device=DEV)
    held, f = s.held.long(), s.count.long()
    in_use = column < held[:, None]                                   # what the source holds, and by whom first
    page, row = s.table.long()[in_use], torch.arange(B, device=DEV)[:, None].expand(B, width)[in_use]
    first = torch.full((num_pages,), none, device=DEV, dtype=torch.long).scatter_reduce(0, page, row, "amin")
    parents = s.parents.long()
    lens = torch.where(parents >= 0, s.lens.long(), 0)
    full, part = lens // P, lens % P
    need = full + (part > 0)
    new = s.table.long()[parents.clamp(min=0)]
    user = torch.arange(len(lens), device=DEV)
    shared = new[column < full[:, None]]
    heir = torch.full((num_pages,), none, device=DEV, dtype=torch.long).scatter_(0, shared, -1)
    has_part = part > 0
    last = new[user, full.clamp(max=width - 1)].clamp(min=0)
    heir = heir.scatter_reduce(0, last[has_part], user[has_part], "amin")
    copies = has_part & (heir[last] != user)
    rank = copies.long().cumsum(0) - 1
    fresh = s.free.long()[(f - 1 - rank).clamp(min=0)]
    count = f - copies.sum()
    new[user[copies], full[copies]] = fresh[copies]
    s.new_table.copy_(torch.where(column < need[:, None], new, s.new_table.long()))
    s.new_held.copy_(need)
    given = page[(heir[page] == none) & (first[page] == row)]
    stack = torch.arange(num_pages, device=DEV)
    kept = torch.where(stack < count, s.free.long(), s.new_free.long())
    kept[count + torch.arange(given.numel(), device=DEV)] = given
    s.new_free.copy_(kept)
    s.new_count.copy_(count + given.numel())
    who = torch.repeat_interleave(user[copies], part[copies])
    at = torch.arange(who.numel(), device=DEV) - torch.repeat_interleave(part[copies].cumsum(0) - part[copies], part[copies])
    for x in (s.k, s.v):
        flat = x.view(x.shape[0], -1, *x.shape[3:])
        flat[:, fresh[who] * P + at] = flat[:, last[who] * P + at]


def exact(case, seed):
    """The definitions in 64 bits: rotations as complex products, softmax over whole rows, forks page by page on the host."""
    if case["kind"] == "lm" and work(case)["flops"] > 6e12:
        return None
    s = prepare(case, seed)
    return {"norm": _exact_norm, "tree": _exact_tree, "logprobs": _exact_logprobs, "lm": _exact_lm,
            "fork": _exact_fork}[case["kind"]](s)


def _exact_turn(x, w, pos):
    d = x.shape[-1]
    x = x.double()
    x = w.double() * x / (x.pow(2).sum(-1, keepdim=True) / d + EPS).sqrt()
    freq = torch.tensor([ROPE_BASE ** (-2.0 * j / d) for j in range(d // 2)], dtype=torch.float64, device=DEV)
    unit = torch.polar(torch.ones_like(pos)[:, None] * torch.ones_like(freq), pos[:, None] * freq)
    z = torch.complex(x[..., :d // 2], x[..., d // 2:]) * unit[:, None, :]
    return torch.cat([z.real, z.imag], -1)


def _exact_norm(s):
    n, hkv, d = s.off[-1], s.case["hkv"], s.case["d"]
    pos = torch.cat([torch.arange(c, c + m, device=DEV, dtype=torch.float64) for c, m in zip(s.ctx, s.new)])
    q, k, v = s.q_out.double(), s.k.double(), s.v.double()
    q[:n] = _exact_turn(s.q[:n], s.wq, pos)
    turned = _exact_turn(s.kn[:n], s.wk, pos)
    for b in range(len(s.new)):
        r = _rows(s, b, s.ctx[b], s.ctx[b] + s.new[b])
        k.view(-1, hkv, d)[r] = turned[s.off[b]:s.off[b + 1]]
        v.view(-1, hkv, d)[r] = s.vn[s.off[b]:s.off[b + 1]].double()
    return {"q": q, "k": k, "v": v}


def _exact_tree(s):
    L, hkv, d = s.k.shape[0], s.case["hkv"], s.case["d"]
    q, k, v = s.q_out.double(), s.k.double(), s.v.double()
    positions = []
    for b, (c, n) in enumerate(zip(s.ctx, s.new)):
        depth = []
        for i in range(n):
            p = s.parents_host[s.off[b] + i]
            depth.append(0 if p < 0 else depth[p] + 1)
        positions += [c + x for x in depth]
    pos = torch.tensor(positions, dtype=torch.float64, device=DEV)
    for l in range(L):
        q[l] = _exact_turn(s.q[l], s.wq[l], pos)
        turned = _exact_turn(s.kn[l], s.wk[l], pos)
        for b in range(len(s.new)):
            r = _rows(s, b, s.ctx[b], s.ctx[b] + s.new[b])
            k[l].view(-1, hkv, d)[r] = turned[s.off[b]:s.off[b + 1]]
            v[l].view(-1, hkv, d)[r] = s.vn[l, s.off[b]:s.off[b + 1]].double()
    return {"q": q, "k": k, "v": v, "positions": np.asarray(positions, np.int32)}


def _exact_rows(s, logits):
    """logits(r) is row block r's 64-bit logits."""
    n, k = s.case["rows"], s.case["k"]
    logprob, entropy = torch.zeros(n, dtype=torch.float64, device=DEV), torch.zeros(n, dtype=torch.float64, device=DEV)
    idx = torch.zeros((n, k), dtype=torch.int32, device=DEV)
    val = torch.zeros((n, k), dtype=torch.float64, device=DEV)
    step = max(1, (1 << 25) // s.case["vocab"])
    for r0 in range(0, n, step):
        r = slice(r0, min(n, r0 + step))
        x = logits(r)
        p = torch.log_softmax(x / s.case["temperature"], -1)
        logprob[r] = p.gather(1, s.tokens[r].long()[:, None])[:, 0]
        entropy[r] = -(p.exp() * p.masked_fill(p == -math.inf, 0.0)).sum(-1)
        if k:
            order = torch.sort(x, dim=-1, descending=True, stable=True).indices[:, :k]
            idx[r], val[r] = order.to(torch.int32), p.gather(1, order)
    return {"logprob": logprob, "entropy": entropy, "top_idx": idx, "top_val": val}


def _exact_logprobs(s):
    return _exact_rows(s, lambda r: s.logits[r].double())


def _exact_lm(s):
    w = s.weight.double()
    return _exact_rows(s, lambda r: s.hidden[r].double() @ w.t())


def _exact_fork(s):
    table, held, free, count, parents, lens = s.host
    P = s.case["page"]
    k, v = s.k.clone(), s.v.clone()
    new_table = s.new_table.cpu().numpy().copy()
    new_free = s.new_free.cpu().numpy().copy()
    stack = [int(x) for x in free[:count]]
    whole, heir = set(), {}
    for b, (p, n) in enumerate(zip(parents, lens)):
        if p >= 0:
            whole.update(int(x) for x in table[p, :n // P])
            if n % P:
                heir.setdefault(int(table[p, n // P]), b)
    new_held = []
    for b, (p, n) in enumerate(zip(parents, lens)):
        if p < 0:
            new_held.append(0)
            continue
        new_table[b, :n // P] = table[p, :n // P]
        if n % P:
            page = int(table[p, n // P])
            if page in whole or heir[page] != b:
                fresh = stack.pop()
                k[:, fresh, :n % P], v[:, fresh, :n % P] = k[:, page, :n % P], v[:, page, :n % P]
                page = fresh
            new_table[b, n // P] = page
        new_held.append(-(-n // P))
    gone = set(whole) | set(heir)
    for b, h in enumerate(held):
        for x in table[b, :h]:
            if int(x) not in gone:
                gone.add(int(x))
                stack.append(int(x))
    new_free[:len(stack)] = stack
    as_i32 = lambda x: np.asarray(x, np.int32)
    return {"k": k, "v": v, "block_table": new_table, "held": as_i32(new_held), "free_pages": new_free,
            "free_count": as_i32([len(stack)])}
