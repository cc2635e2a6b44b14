"""Performance cases of the prompt path: slots and block tables, the rotary append, prompt attention.

A serving loop admits a packed batch of requests (whole prompts, chunks of prompts, or one token
each) as follows: `prompt_slots` gives every request the pages its length needs and every new token
its cache row and position; per layer `prompt_rope_append` rotates Q and K and writes K and V into
those rows, and `prompt_attention` attends, causally, from the new tokens to everything before them.
`listed()` holds fixed sizes, `draw()` further ones of the same ranges.  Inputs are drawn on the GPU
from the seed: Q, K, V ~ N(0, 1).  `plain` forms are elementary torch operations in 32 bits.
"""
from __future__ import annotations

import math
import random

import numpy as np
import torch

own = False

DEV = "cuda"
ROPE_BASE = 500000.0
MAX_FLOPS = 4.4e12      # of one pass: the largest listed case (attn_prompt_16384)
MAX_TOKENS = 262144


def listed():
    return [
        # one decoded token for each of eight ragged requests over 16-token pages, 32q/8kv
        {"name": "attn_decode_8", "kind": "attn", "dtype": "bf16", "hq": 32, "hkv": 8, "d": 128, "page": 16, "batch": 8,
         "new": 1, "ctx": 4096, "ragged": True, "mix": 1, "pad": 0},
        # a continuous batch: ragged prompts between one token and a thousand, padded to a captured size
        {"name": "attn_ragged_prompts", "kind": "attn", "dtype": "bf16", "hq": 32, "hkv": 8, "d": 128, "page": 16,
         "batch": 8, "new": 1021, "ctx": 0, "ragged": True, "mix": 2, "pad": 37},
        # a whole prompt of a 7B MHA model's layer
        {"name": "attn_prompt_mha", "kind": "attn", "dtype": "bf16", "hq": 32, "hkv": 32, "d": 128, "page": 0, "batch": 1,
         "new": 2047, "ctx": 0, "ragged": False, "mix": 0, "pad": 0},
        # a whole prompt of an 8B GQA model's layer
        {"name": "attn_prompt_8192", "kind": "attn", "dtype": "bf16", "hq": 32, "hkv": 8, "d": 128, "page": 0, "batch": 1,
         "new": 8192, "ctx": 0, "ragged": False, "mix": 0, "pad": 0},
        # a small chunk late in a long document: few rows, many keys
        {"name": "attn_chunk_long", "kind": "attn", "dtype": "bf16", "hq": 64, "hkv": 8, "d": 128, "page": 64, "batch": 1,
         "new": 61, "ctx": 32707, "ragged": False, "mix": 0, "pad": 0},
        # the largest: half a long-context prompt at once, 64q/8kv
        {"name": "attn_prompt_16384", "kind": "attn", "dtype": "bf16", "hq": 64, "hkv": 8, "d": 128, "page": 128,
         "batch": 1, "new": 16384, "ctx": 0, "ragged": False, "mix": 0, "pad": 0},
        # prompts of a small model kept in fp32
        {"name": "attn_f32", "kind": "attn", "dtype": "f32", "hq": 8, "hkv": 8, "d": 64, "page": 0, "batch": 3, "new": 256,
         "ctx": 0, "ragged": True, "mix": 3, "pad": 0},
        # a decoding batch's rotary encoding and append, from fused QKV rows
        {"name": "append_decode_8", "kind": "append", "dtype": "bf16", "hq": 32, "hkv": 8, "d": 128, "page": 16, "batch": 8,
         "new": 1, "ctx": 4096, "ragged": True, "mix": 1, "pad": 0},
        # a long prompt's
        {"name": "append_prompt_8192", "kind": "append", "dtype": "bf16", "hq": 32, "hkv": 8, "d": 128, "page": 0,
         "batch": 1, "new": 8192, "ctx": 0, "ragged": False, "mix": 0, "pad": 0},
        # a decoding batch's pages: most requests stay in their last page, some need one more
        {"name": "slots_decode_256", "kind": "slots", "page": 16, "batch": 256, "new": 1, "ctx": 4096, "ragged": True,
         "mix": 4, "pad": 0},
        # admission of many prompts beside requests that have finished
        {"name": "slots_admit", "kind": "slots", "page": 16, "batch": 96, "new": 4096, "ctx": 0, "ragged": True, "mix": 5,
         "pad": 301},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["attn", "attn", "attn", "append", "slots"])
    while True:
        c = {"kind": kind, "page": rng.choice([0, 16, 32, 64, 128]), "batch": 1 if rng.random() < 0.4 else _log(rng, 2, 64),
             "new": 1 if rng.random() < 0.2 else _log(rng, 2, 16384), "ctx": 0 if rng.random() < 0.4 else _log(rng, 1, 32768),
             "ragged": rng.random() < 0.7, "mix": rng.randrange(1 << 20), "pad": rng.choice([0, 0, rng.randrange(1, 200)])}
        if kind == "slots":
            c["page"] = rng.choice([16, 32, 64, 128])
            c["batch"] = _log(rng, 1, 1024)
        else:
            c["dtype"] = "bf16" if rng.random() < 0.8 else "f32"
            if c["dtype"] == "bf16":
                c["hq"], c["hkv"] = rng.choice([(32, 32), (32, 8), (64, 8), (16, 2), (28, 4), (40, 8)])
                c["d"] = 128
            else:
                c["hq"], c["hkv"] = rng.choice([(8, 8), (16, 16), (32, 8)])
                c["d"] = rng.choice([32, 64, 128])
                c["new"], c["ctx"] = min(c["new"], 2048), min(c["ctx"], 4096)
        ctx, new = _lengths(c)
        if sum(new) > MAX_TOKENS or (kind != "slots" and sum(ctx) + sum(new) > MAX_TOKENS):
            continue
        if kind == "attn" and work(c)["flops"] > (MAX_FLOPS if c["dtype"] == "bf16" else MAX_FLOPS / 40):
            continue
        return c


def _lengths(case):
    """Contexts and numbers of new tokens, host lists: a function of the case alone."""
    rng = random.Random(case["mix"])
    ctx, new = [], []
    for b in range(case["batch"]):
        if case["ragged"]:
            new.append(case["new"] if b == 0 else _log(rng, 1, case["new"]))
            ctx.append(case["ctx"] if b == 0 or case["ctx"] == 0 else _log(rng, max(1, case["ctx"] // 4), case["ctx"]))
        else:
            new.append(case["new"])
            ctx.append(case["ctx"])
        if case["kind"] == "slots" and rng.random() < 0.15:   # a finished request, whose pages come back
            new[-1] = ctx[-1] = 0
    if sum(new) == 0:
        new[0] = 1
    return ctx, new


def _held(case):
    """Pages that every request of a slots case holds before the call."""
    ctx, new = _lengths(case)
    rng = random.Random(case["mix"] + 1)
    held = []
    for c, n in zip(ctx, new):
        h = -(-c // case["page"])
        if c == 0 and n == 0:
            h = -(-max(case["ctx"], case["new"]) // case["page"]) // 2
        elif c and rng.random() < 0.1:   # pages reserved for a rejected draft
            h += rng.randrange(1, 4)
        held.append(h)
    return held


def _offsets(new):
    return [0] + [int(x) for x in np.cumsum(new)]


def _size(dtype):
    return 2 if dtype == "bf16" else 4


def work(case):
    ctx, new = _lengths(case)
    N, B = sum(new), len(new)
    if case["kind"] == "slots":
        need = [-(-(c + n) // case["page"]) for c, n in zip(ctx, new)]
        moved = sum(abs(n - h) for n, h in zip(need, _held(case)))
        return {"bytes": 4 * (B + 1) + 12 * B + 8 * moved + 8 * (N + case["pad"]), "flops": 2 * N}
    e, d, hq, hkv = _size(case["dtype"]), case["d"], case["hq"], case["hkv"]
    if case["kind"] == "append":
        return {"bytes": N * (2 * hq + 4 * hkv) * d * e + 8 * N, "flops": 3 * N * (hq + hkv) * d}
    pairs = sum(n * c + n * (n + 1) // 2 for c, n in zip(ctx, new))
    return {"bytes": 2 * N * hq * d * e + 2 * (sum(ctx) + N) * hkv * d * e, "flops": 4 * d * hq * pairs}


class State:
    pass


def prepare(case, seed):
    s = State()
    s.case = case
    ctx, new = _lengths(case)
    s.ctx, s.new, s.off = ctx, new, _offsets(new)
    g = torch.Generator(device=DEV).manual_seed(seed)
    host = np.random.default_rng(seed)
    i32 = dict(dtype=torch.int32, device=DEV)
    B, N, page = len(new), s.off[-1] + case["pad"], case["page"]
    s.N = N
    s.token_offsets = torch.tensor(s.off, **i32)
    s.ctx_lens = torch.tensor(ctx, **i32)
    s.slots = torch.full((N,), -1, **i32)
    s.positions = torch.full((N,), -1, **i32)
    s.status = torch.zeros(1, **i32)
    if case["kind"] == "slots":
        need = [-(-(c + n) // page) for c, n in zip(ctx, new)]
        held = _held(case)
        width = max(max(need), max(held)) + 2
        num_pages = sum(max(a, b) for a, b in zip(need, held)) + 17
        perm = host.permutation(num_pages).astype(np.int32)
        table = np.full((B, width), -1, np.int32)
        at = 0
        for b, h in enumerate(held):
            table[b, :h] = perm[at:at + h]
            at += h
        free = np.full(num_pages, -1, np.int32)
        free[:num_pages - at] = perm[at:]
        s.block_table, s.free_pages = torch.tensor(table, **i32), torch.tensor(free, **i32)
        s.free_count, s.held = torch.tensor([num_pages - at], **i32), torch.tensor(held, **i32)
        s.new_held, s.new_free_count = torch.zeros_like(s.held), torch.zeros_like(s.free_count)
        s.host = (table, free, num_pages - at, held)
        k = torch.zeros((1, num_pages, page, 1, 8), dtype=torch.bfloat16, device=DEV)   # one layer of a small cache
        if own:   # descriptions of the buffers above, which a program keeps
            from paper_2607_10661_gb300 import ptd
            s.cache = ptd.KVCache(k, k.clone(), 1, 8, page, s.block_table)
            s.prompt = ptd.Prompt(s.token_offsets, s.ctx_lens, N, max(new), max(ctx))
            s.pages = ptd.PagePool(s.free_pages, s.free_count, s.held, s.new_held, s.new_free_count)
        return s
    t = torch.bfloat16 if case["dtype"] == "bf16" else torch.float32
    hq, hkv, d = case["hq"], case["hkv"], case["d"]
    longest = max(c + n for c, n in zip(ctx, new))
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
        shape = (1, num_pages, page, hkv, d)
    else:
        s.block_table = None
        shape = (1, B, longest + 5, hkv, d)
    s.k = torch.randn(shape, generator=g, device=DEV, dtype=torch.float32).to(t)
    s.v = torch.randn(shape, generator=g, device=DEV, dtype=torch.float32).to(t)
    if case["kind"] == "attn":
        s.q = torch.randn((N, hq, d), generator=g, device=DEV, dtype=torch.float32).to(t)
        s.out = torch.zeros((N, hq, d), dtype=t, device=DEV)
    else:
        qkv = torch.randn((N, (hq + 2 * hkv) * d), generator=g, device=DEV, dtype=torch.float32).to(t)
        s.q = qkv[:, :hq * d].view(N, hq, d)
        s.kn = qkv[:, hq * d:(hq + hkv) * d].view(N, hkv, d)
        s.vn = qkv[:, (hq + hkv) * d:].view(N, hkv, d)
        s.q_out = torch.zeros((N, hq, d), dtype=t, device=DEV)
        for b in range(B):
            s.slots[s.off[b]:s.off[b + 1]] = _rows(s, b, ctx[b], ctx[b] + new[b]).to(torch.int32)
            s.positions[s.off[b]:s.off[b + 1]] = torch.arange(ctx[b], ctx[b] + new[b], **i32)
    if own:   # descriptions of the buffers above, and the scratch, which a program keeps
        from paper_2607_10661_gb300 import ptd
        s.cache = ptd.KVCache(s.k, s.v, hkv, d, page, s.block_table)
        s.prompt = ptd.Prompt(s.token_offsets, s.ctx_lens, N, max(new), max(ctx))
        n = ptd.prompt_attention_workspace_size(s.prompt, s.cache, hq) if case["kind"] == "attn" else 0
        s.workspace = torch.empty(n, dtype=torch.uint8, device=DEV) if n else None
    return s


def _rows(s, b, lo, hi):
    """Cache rows of request b's positions lo .. hi - 1."""
    p = torch.arange(lo, hi, device=DEV)
    if s.block_table is None:
        return b * s.k.shape[2] + p
    page = s.case["page"]
    return s.block_table[b].long()[p // page] * page + p % page


def run(s):
    kind = s.case["kind"]
    if own:
        from paper_2607_10661_gb300 import ptd
        if kind == "slots":
            ptd.prompt_slots(s.prompt, s.cache, s.slots, s.positions, s.status, s.pages)
        elif kind == "append":
            ptd.prompt_rope_append(s.prompt, s.cache, 0, s.slots, s.positions, s.q, s.kn, s.vn, s.q_out, ROPE_BASE, s.status)
        else:
            ptd.prompt_attention(s.prompt, s.cache, 0, s.q, s.out, s.status, workspace=s.workspace)
    elif kind == "slots":
        _plain_slots(s)
    elif kind == "append":
        _plain_append(s)
    else:
        _plain_attention(s)
    if kind == "slots":
        return {"block_table": s.block_table, "free_pages": s.free_pages, "new_held": s.new_held,
                "new_free_count": s.new_free_count, "slots": s.slots, "positions": s.positions}
    if kind == "append":
        return {"q": s.q_out, "k": s.k, "v": s.v}
    return s.out


def _plain_slots(s):
    page = s.case["page"]
    off, ctx, held, f = s.token_offsets.long(), s.ctx_lens.long(), s.held.long(), s.free_count.long()
    new = off[1:] - off[:-1]
    need = (ctx + new + page - 1) // page
    gives, takes = (held - need).clamp(min=0), (need - held).clamp(min=0)
    G, T = gives.sum(), takes.sum()
    seqs = torch.arange(len(s.new), device=DEV)
    gb = torch.repeat_interleave(seqs, gives)            # the request and index of every page given and taken
    gi = torch.arange(gb.numel(), device=DEV) - (gives.cumsum(0) - gives)[gb] + need[gb]
    tb = torch.repeat_interleave(seqs, takes)
    rank = torch.arange(tb.numel(), device=DEV)
    ti = rank - (takes.cumsum(0) - takes)[tb] + held[tb]
    given = s.block_table[gb, gi]
    stack = torch.cat([given.flip(0), s.free_pages.index_select(0, (f - 1 - torch.arange(s.free_pages.numel(), device=DEV)).clamp(min=0))])
    s.block_table[tb, ti] = stack[rank]
    keep = torch.arange(gb.numel(), device=DEV)
    keep = keep[keep < G - T]
    s.free_pages[f + keep] = given[keep]
    s.new_held.copy_(need)
    s.new_free_count.copy_(f + G - T)
    b = torch.repeat_interleave(seqs, new)
    pos = torch.arange(b.numel(), device=DEV) - off[:-1][b] + ctx[b]
    s.slots.fill_(-1)
    s.positions.fill_(-1)
    s.slots[:b.numel()] = (s.block_table[b, pos // page] * page + pos % page).to(torch.int32)
    s.positions[:b.numel()] = pos.to(torch.int32)


def _plain_append(s):
    d = s.case["d"]
    n = s.off[-1]   # the rows behind the last request stay as they were
    j = torch.arange(d // 2, device=DEV, dtype=torch.float64)
    angle = s.positions[:n, None].double() * torch.pow(torch.tensor(ROPE_BASE, device=DEV, dtype=torch.float64), -2.0 * j / d)
    c, sn = angle.cos().float()[:, None, :], angle.sin().float()[:, None, :]

    def turn(x):
        a, b = x[:n, :, :d // 2].float(), x[:n, :, d // 2:].float()
        return torch.cat([a * c - b * sn, a * sn + b * c], -1).to(x.dtype)

    s.q_out[:n] = turn(s.q)
    rows = s.slots[:n].long()
    s.k.view(-1, *s.k.shape[3:])[rows] = turn(s.kn)
    s.v.view(-1, *s.v.shape[3:])[rows] = s.vn[:n]


def _plain_attention(s):
    hq, hkv, d = s.case["hq"], s.case["hkv"], s.case["d"]
    kf, vf = s.k.view(-1, hkv, d), s.v.view(-1, hkv, d)
    B, lens = len(s.new), [c + n for c, n in zip(s.ctx, s.new)]
    # all requests at once, padded to the longest, unless that is over twice the work
    together = B * max(s.new) * max(lens) <= 2 * sum(n * m for n, m in zip(s.new, lens))
    for seqs in [list(range(B))] if together else [[b] for b in range(B)]:
        G, n, m = len(seqs), max(s.new[b] for b in seqs), max(lens[b] for b in seqs)
        ids = torch.tensor(seqs, device=DEV) if G < B else torch.arange(B, device=DEV)
        off, ctx = s.token_offsets.long()[ids, None], s.ctx_lens.long()[ids, None]
        new = s.token_offsets.long()[ids + 1, None] - off
        p = torch.arange(m, device=DEV)[None, :].minimum(ctx + new - 1)
        rows = ids[:, None] * s.k.shape[2] + p if s.block_table is None else _paged_rows(s, ids, p)
        k, v = kf[rows].float().permute(0, 2, 3, 1), vf[rows].float().permute(0, 2, 1, 3)   # [G, hkv, d, m], [G, hkv, m, d]
        step = max(1, min(n, (1 << 28) // (G * hq * m)))
        for i0 in range(0, n, step):
            i1 = min(n, i0 + step)
            keys = min(m, max(s.ctx[b] for b in seqs) + i1)
            i = torch.arange(i0, i1, device=DEV)[None, :]
            token = off + i.minimum(new - 1)
            q = s.q[token].float().view(G, i1 - i0, hkv, hq // hkv, d).permute(0, 2, 3, 1, 4)
            x = torch.matmul(q.reshape(G, hkv, -1, d), k[..., :keys]).mul_(1.0 / math.sqrt(d))
            x = x.view(G, hkv, hq // hkv, i1 - i0, keys)
            hidden = torch.arange(keys, device=DEV) > (ctx + i)[:, :, None]
            x.masked_fill_(hidden[:, None, None], -math.inf)
            x = (x - x.amax(-1, keepdim=True)).exp_()
            o = torch.matmul(x.view(G, hkv, -1, keys), v[:, :, :keys]).view(G, hkv, hq // hkv, i1 - i0, d)
            o = (o / x.sum(-1, keepdim=True)).permute(0, 3, 1, 2, 4).reshape(G, i1 - i0, hq, d).to(s.out.dtype)
            there = i < new
            s.out[token[there]] = o[there]


def _paged_rows(s, ids, p):
    page = s.case["page"]
    return s.block_table.long()[ids[:, None], p // page] * page + p % page


def exact(case, seed):
    """The definition in 64 bits: allocation page by page on the host, rotations as complex products, attention
    one KV head and block of queries at a time."""
    if case["kind"] == "attn" and work(case)["flops"] > 9e12:
        return None
    s = prepare(case, seed)
    if case["kind"] == "slots":
        return _exact_slots(s)
    n = s.off[-1]
    hq, hkv, d = case["hq"], case["hkv"], case["d"]
    if case["kind"] == "append":
        freq = torch.tensor([ROPE_BASE ** (-2.0 * j / d) for j in range(d // 2)], dtype=torch.float64, device=DEV)
        pos = torch.cat([torch.arange(c, c + m, device=DEV, dtype=torch.float64) for c, m in zip(s.ctx, s.new)])
        unit = torch.polar(torch.ones_like(pos)[:, None] * torch.ones_like(freq), pos[:, None] * freq)
        def turn(x):
            z = torch.complex(x[:n, :, :d // 2].double(), x[:n, :, d // 2:].double()) * unit[:, None, :]
            return torch.cat([z.real, z.imag], -1)
        q, k, v = s.q_out.double(), s.k.double(), s.v.double()
        q[:n] = turn(s.q)
        for b in range(len(s.new)):
            r = _rows(s, b, s.ctx[b], s.ctx[b] + s.new[b])
            k.view(-1, hkv, d)[r] = turn(s.kn)[s.off[b]:s.off[b + 1]]
            v.view(-1, hkv, d)[r] = s.vn[s.off[b]:s.off[b + 1]].double()
        return {"q": q, "k": k, "v": v}
    out = torch.zeros((s.N, hq, d), dtype=torch.float64, device=DEV)
    group = hq // hkv
    for b in range(len(s.new)):
        c, m = s.ctx[b], s.new[b]
        for h in range(hkv):
            k = s.k.view(-1, hkv, d)[_rows(s, b, 0, c + m), h].double()
            v = s.v.view(-1, hkv, d)[_rows(s, b, 0, c + m), h].double()
            step = max(1, (1 << 26) // (group * (c + m)))
            for i0 in range(0, m, step):
                i1 = min(m, i0 + step)
                q = s.q[s.off[b] + i0:s.off[b] + i1, h * group:(h + 1) * group].double()
                x = torch.einsum("ngd,kd->ngk", q, k[:c + i1]) / math.sqrt(d)
                own_pos = torch.arange(c + i0, c + i1, device=DEV)
                x = torch.where(torch.arange(c + i1, device=DEV) <= own_pos[:, None, None], x, -math.inf)
                w = torch.softmax(x, -1)
                out[s.off[b] + i0:s.off[b] + i1, h * group:(h + 1) * group] = torch.einsum("ngk,kd->ngd", w, v[:c + i1])
    return out


def _exact_slots(s):
    table, free, count, held = (x.copy() if isinstance(x, np.ndarray) else x for x in s.host)
    page = s.case["page"]
    stack = [int(x) for x in free[:count]]
    need = [-(-(c + n) // page) for c, n in zip(s.ctx, s.new)]
    for b, (h, w) in enumerate(zip(held, need)):
        stack += [int(x) for x in table[b, w:h]]
    for b, (h, w) in enumerate(zip(held, need)):
        for i in range(h, w):
            table[b, i] = stack.pop()
    if len(stack) > count:
        free[count:len(stack)] = stack[count:]
    slots, positions = np.full(s.N, -1, np.int32), np.full(s.N, -1, np.int32)
    for b in range(len(need)):
        for i in range(s.new[b]):
            p = s.ctx[b] + i
            slots[s.off[b] + i] = table[b, p // page] * page + p % page
            positions[s.off[b] + i] = p
    as_i32 = lambda x: np.asarray(x, np.int32)
    return {"block_table": table, "free_pages": free, "new_held": as_i32(need),
            "new_free_count": as_i32([len(stack)]), "slots": slots, "positions": positions}
