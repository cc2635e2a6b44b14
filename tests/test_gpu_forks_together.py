"""Forks, norms with the append and log probabilities as they are used: with the page pool and the attention, captured and
replayed, on streams of their own, at offsets past 32 bits, through both of the binding's paths."""
import math

import numpy as np
import pytest
import torch

import oracle
from paper_2607_10661_gb300 import ptd

pytestmark = pytest.mark.gpu
DEV = "cuda"
BF16, F32 = torch.bfloat16, torch.float32
I32 = dict(dtype=torch.int32, device=DEV)


@pytest.fixture(scope="module", autouse=True)
def _built():
    import __graft_entry__

    __graft_entry__.build()


def _empty_set(batch, width, num_pages):
    return ptd.PageSet(torch.full((batch, width), -1, **I32), torch.zeros(batch, **I32), torch.full((num_pages,), -1, **I32),
                       torch.zeros(1, **I32))


def _fork_space(cache, a, b):
    return torch.empty(ptd.page_fork_workspace_size(cache, a, b), dtype=torch.uint8, device=DEV)


@pytest.mark.parametrize("seed,page,most", [(0, 16, 12), (1, 32, 40), (2, 128, 7)])
def test_random_forks_and_growth(seed, page, most):
    """Sequences grow (pages from prompt_slots), fork, are cut and end, at random, some steps long: every page is held or
    free, and once only among the free ones; every sequence's K and V rows are what was written to it and its ancestors."""
    rng = np.random.default_rng(seed)
    L, hkv, d, width, num = 2, 1, 8, 24, 24 * most
    k, v = (torch.zeros((L, num, page, hkv, d), dtype=F32, device=DEV) for _ in range(2))
    now = _empty_set(most, width, num)
    now.free_pages.copy_(torch.tensor(rng.permutation(num), **I32))
    now.free_count.fill_(num)
    status = torch.zeros(1, **I32)
    want = [[] for _ in range(most)]   # the values of every position
    fresh = 1.0
    for step in range(14):
        # growth: prompt_slots in place, then values into the new slots
        new = [int(rng.integers(0, 2 * page)) if len(w) + 2 * page < (width - 1) * page and rng.random() < 0.8 else 0 for w in want]
        cache = ptd.KVCache(k, v, hkv, d, page, now.block_table)
        N = sum(new) + 1
        off = torch.tensor(np.concatenate([[0], np.cumsum(new)]), **I32)
        prompt = ptd.Prompt(off, torch.tensor([len(w) for w in want], **I32), N, 2 * page, width * page)
        pool = ptd.PagePool(now.free_pages, now.free_count, now.held, torch.empty_like(now.held), torch.empty_like(now.free_count))
        slots, pos = torch.empty(N, **I32), torch.empty(N, **I32)
        ptd.prompt_slots(prompt, cache, slots, pos, status, pool)
        now.held.copy_(pool.new_held)
        now.free_count.copy_(pool.new_free_count)
        values = torch.arange(N, device=DEV, dtype=F32) + fresh
        fresh += N
        at = slots[:N - 1].long()
        for l in range(L):
            k[l].view(-1, hkv, d)[at] = (values[:N - 1] * (l + 1))[:, None, None].expand(-1, hkv, d)
            v[l].view(-1, hkv, d)[at] = (-values[:N - 1] * (l + 1))[:, None, None].expand(-1, hkv, d)
        host = values.tolist()
        i = 0
        for b, n in enumerate(new):
            want[b] = want[b] + host[i:i + n]
            i += n
        # a fork into a batch of another set
        parents = [int(rng.integers(-1, most)) for _ in range(most)]
        lens = [0 if p < 0 else (len(want[p]) if rng.random() < 0.7 else int(rng.integers(0, len(want[p]) + 1))) for p in parents]
        then = _empty_set(most, width, num)
        ptd.page_fork(cache, now, then, torch.tensor(parents, **I32), torch.tensor(lens, **I32), _fork_space(cache, now, then), status)
        now, want = then, [[] if p < 0 else want[p][:n] for p, n in zip(parents, lens)]
        assert int(status) == 0
        table, held = now.block_table.tolist(), now.held.tolist()
        assert held == [-(-len(w) // page) for w in want]
        free = now.free_pages[:int(now.free_count)].tolist()
        in_use = {x for r, h in zip(table, held) for x in r[:h]}
        assert len(set(free)) == len(free) and not in_use & set(free) and len(in_use) + len(free) == num
        for b, w in enumerate(want):
            for own in table[b][len(w) // page:held[b]]:   # a partial page is its sequence's alone
                assert sum(own in r[:h] for r, h in zip(table, held)) == 1
            if not w:
                continue
            p = torch.arange(len(w), device=DEV)
            rows = now.block_table[b].long()[p // page] * page + p % page
            for l in range(L):
                got = k[l].view(-1, hkv, d)[rows]
                exp = (torch.tensor(w, device=DEV) * (l + 1))[:, None, None].expand(-1, hkv, d)
                assert torch.equal(got, exp) and torch.equal(v[l].view(-1, hkv, d)[rows], -exp)


def _normed(x, w, pos, base, eps):
    x, d = x.double(), x.shape[-1]
    y = x * w.double() / (x.square().mean(-1, keepdim=True) + eps).sqrt()
    a = torch.tensor(pos, dtype=torch.float64, device=DEV)[:, None] * base ** (-2.0 * torch.arange(d // 2, device=DEV, dtype=torch.float64) / d)
    c, s = a.cos()[:, None], a.sin()[:, None]
    p, q = y[..., :d // 2], y[..., d // 2:]
    return torch.cat([p * c - q * s, p * s + q * c], -1)


def test_beams_together():
    """Two requests, their prompts once, then beams over shared pages: slots, norms with the append, attention, log
    probabilities with alternatives from hidden states, forks.  A small model of two layers against the same in 64 bits with
    every beam on its own.  Rounding is followed: the 64-bit side rounds to bf16 where the operators do, so that attention
    outputs differ by the steps of their own tolerance (2^-7 of the outputs' size) and scores by little more than those of
    the log probabilities; the beams themselves are picked by the operators."""
    g = torch.Generator(device=DEV).manual_seed(5)
    L, hq, hkv, d, page, V, beams, base, eps = 2, 4, 2, 128, 16, 1000, 3, 1e4, 1e-6
    B, width, num = 2 * beams, 12, 80
    E = (torch.randn((V, hq * d), generator=g, device=DEV) * 0.5).to(BF16)                       # embeddings and the head
    wq = [(torch.randn((hq * d, hq * d), generator=g, device=DEV) / math.sqrt(hq * d)).to(BF16) for _ in range(L)]
    wkv = [(torch.randn((hq * d, 2 * hkv * d), generator=g, device=DEV) / math.sqrt(hq * d)).to(BF16) for _ in range(L)]
    nq, nk = ((1 + 0.2 * torch.randn((L, d), generator=g, device=DEV)).to(BF16) for _ in range(2))
    k, v = (torch.full((L, num, page, hkv, d), float("nan"), dtype=BF16, device=DEV) for _ in range(2))
    now, status = _empty_set(2, width, num), torch.zeros(1, **I32)
    now.free_pages.copy_(torch.arange(num, **I32))
    now.free_count.fill_(num)
    tokens = [torch.randint(0, V, (n,), generator=g, device=DEV).tolist() for n in (37, 20)]
    ctx, new = [0, 0], [t[:] for t in tokens]
    score = None
    for step in range(5):
        cache = ptd.KVCache(k, v, hkv, d, page, now.block_table)
        N = sum(map(len, new))
        off_h = np.concatenate([[0], np.cumsum([len(x) for x in new])])
        prompt = ptd.Prompt(torch.tensor(off_h, **I32), torch.tensor(ctx, **I32), N, max(map(len, new)), 100)
        pool = ptd.PagePool(now.free_pages, now.free_count, now.held, torch.empty_like(now.held), torch.empty_like(now.free_count))
        slots, pos = torch.empty(N, **I32), torch.empty(N, **I32)
        ptd.prompt_slots(prompt, cache, slots, pos, status, pool)
        now.held.copy_(pool.new_held)
        now.free_count.copy_(pool.new_free_count)
        x = E[torch.tensor([t for s in new for t in s], device=DEV)]
        for l in range(L):
            q, kv = (x @ wq[l]).view(N, hq, d), (x @ wkv[l]).view(N, 2 * hkv, d)
            qn, o = torch.empty_like(q), torch.empty_like(q)
            ptd.prompt_norm_rope_append(prompt, cache, l, slots, pos, q, kv[:, :hkv], kv[:, hkv:], qn, nq[l], nk[l], eps, base, status)
            ws = torch.empty(max(16, ptd.prompt_attention_workspace_size(prompt, cache, hq)), dtype=torch.uint8, device=DEV)
            ptd.prompt_attention(prompt, cache, l, qn, o, status, workspace=ws)
            # against 64 bits, every sequence by itself from its own pages
            for b in range(len(new)):
                sl, n = slice(int(off_h[b]), int(off_h[b + 1])), ctx[b] + len(new[b])
                p = torch.arange(n, device=DEV)
                rows = now.block_table[b].long()[p // page] * page + p % page
                kb, vb = (c[l].view(-1, hkv, d)[rows].double() for c in (k, v))
                assert torch.isfinite(kb).all() and torch.equal(vb[ctx[b]:], kv[sl, hkv:].double())
                mine = _normed(kv[sl, :hkv], nk[l], list(range(ctx[b], n)), base, eps)
                assert ((kb[ctx[b]:] - mine).abs() <= mine.abs() * 2.0 ** -8 * 1.01 + 2.0 ** -16).all()
                mine = _normed(q[sl], nq[l], list(range(ctx[b], n)), base, eps)
                assert ((qn[sl].double() - mine).abs() <= mine.abs() * 2.0 ** -8 * 1.01 + 2.0 ** -16).all()
                ref, size = oracle.causal_attention(qn[sl].double().cpu().numpy(), kb.cpu().numpy(), vb.cpu().numpy(), ctx[b])
                assert (np.abs(o[sl].double().cpu().numpy() - ref) <= 2.0 ** -7 * (size + np.abs(ref))).all()
            x = (x + o.view(N, -1)).contiguous()
        last = x[torch.tensor(off_h[1:] - 1, device=DEV)].contiguous()
        S = len(new)
        lp, ent, idx, val = torch.zeros(S, device=DEV), torch.zeros(S, device=DEV), torch.zeros((S, beams), **I32), torch.zeros((S, beams), device=DEV)
        ws = torch.empty(ptd.lm_head_logprobs_workspace_size(S, V, beams), dtype=torch.uint8, device=DEV)
        taken = torch.randint(0, V, (S,), generator=g, device=DEV).to(torch.int32)
        ptd.lm_head_logprobs(last, E, taken, lp, ent, idx, val, ws, status)
        exact = torch.log_softmax(last.double() @ E.double().t(), -1)
        size = float((last.double().abs() @ E.double().abs().t()).max())
        tol = 2 * hq * d * 2.0 ** -23 * size + 2.0 ** -16
        assert ((lp.double() - exact.gather(1, taken.long()[:, None])[:, 0]).abs() <= tol).all()
        assert ((val.double() - exact.gather(1, idx.long())).abs() <= tol).all()
        assert ((val.double() - exact.topk(beams).values).abs() <= tol).all()
        # the same from logits that were written
        logits = (last.float() @ E.float().t()).contiguous()
        other = [torch.zeros_like(t) for t in (lp, ent, idx, val)]
        ptd.token_logprobs(logits, taken, *other, status)
        assert ((other[0] - lp).abs() <= 2 * tol).all() and ((other[1] - ent).abs() <= 2 * tol * (1 + ent)).all()
        # the best beams of each request
        length = [c + len(n) for c, n in zip(ctx, new)]
        total = val if score is None else score[:, None] + val
        per = S // 2
        parents, picked, kept = [], [], []
        for r in range(2):
            best = total[r * per:(r + 1) * per].flatten().topk(beams)
            for s, i in zip(best.values.tolist(), best.indices.tolist()):
                parents.append(r * per + i // beams)
                picked.append([int(idx[r * per + i // beams, i % beams])])
                kept.append(s)
        score = torch.tensor(kept, device=DEV)
        then = _empty_set(B, width, num)
        ptd.page_fork(cache, now, then, torch.tensor(parents, **I32), torch.tensor([length[p] for p in parents], **I32),
                      _fork_space(cache, now, then), status)
        ctx, new, now = [length[p] for p in parents], picked, then
        assert int(status) == 0
        free = now.free_pages[:int(now.free_count)].tolist()
        assert len(set(free) | {x for r, h in zip(now.block_table.tolist(), now.held.tolist()) for x in r[:h]}) == num
    # all but one beam end: their pages come back
    then = _empty_set(1, width, num)
    cache = ptd.KVCache(k, v, hkv, d, page, now.block_table)
    ptd.page_fork(cache, now, then, torch.tensor([2], **I32), torch.tensor([ctx[2]], **I32), _fork_space(cache, now, then), status)
    assert int(then.free_count) == num - -(-ctx[2] // page) and int(status) == 0


def test_trees_with_norms_verify_as_prompts_do():
    """A tree that is a chain, appended with norms, gives the prompt form's rows and queries bit for bit, over forked pages."""
    g = torch.Generator(device=DEV).manual_seed(9)
    hq, hkv, d, page, n = 8, 2, 128, 16, 7
    k, v = (torch.randn((1, 12, page, hkv, d), generator=g, device=DEV).to(BF16) for _ in range(2))
    src = ptd.PageSet(torch.tensor([[3, 1, -1, -1]], **I32), torch.tensor([2], **I32),
                      torch.tensor([0, 2, 4, 5, 6, 7, 8, 9, 10, 11, -1, -1], **I32), torch.tensor([10], **I32))
    dst, status = _empty_set(2, 4, 12), torch.zeros(1, **I32)
    cache = ptd.KVCache(k, v, hkv, d, page, src.block_table)
    ptd.page_fork(cache, src, dst, torch.zeros(2, **I32), torch.tensor([20, 20], **I32), _fork_space(cache, src, dst), status)
    assert dst.block_table[:, :2].tolist() == [[3, 1], [3, 11]]
    cache = ptd.KVCache(k, v, hkv, d, page, dst.block_table)
    q, kn, vn = (torch.randn((2 * n, h, d), generator=g, device=DEV).to(BF16) for h in (hq, hkv, hkv))
    w = (1 + 0.1 * torch.randn((2, d), generator=g, device=DEV)).to(BF16)
    off, ctx = torch.tensor([0, n, 2 * n], **I32), torch.tensor([20, 20], **I32)
    prompt = ptd.Prompt(off, ctx, 2 * n, n, 20)
    slots, pos = torch.empty(2 * n, **I32), torch.empty(2 * n, **I32)
    ptd.prompt_slots(prompt, cache, slots, pos, status)
    out = torch.empty_like(q)
    ptd.prompt_norm_rope_append(prompt, cache, 0, slots, pos, q, kn, vn, out, w[0], w[1], 1e-6, 1e4, status)
    k1, v1 = k.clone(), v.clone()
    tree = ptd.Tree(off, torch.tensor(list(range(-1, n - 1)) * 2, **I32), ctx, n, 20)
    out2, pos2 = torch.empty_like(q)[None], torch.empty(2 * n, **I32)
    ptd.tree_norm_rope_append(tree, cache, 0, q[None], kn[None], vn[None], out2, w[:1], w[1:], 1e-6, 1e4, status, pos2)
    assert torch.equal(out2[0], out) and torch.equal(pos, pos2) and torch.equal(k, k1) and torch.equal(v, v1)
    assert int(status) == 0


def test_captured_forks_and_scores():
    """A fork there and back and the scores of its sequences, captured once and replayed with other parents, lengths,
    logits and tokens; a second graph shares the scratch."""
    rng = np.random.default_rng(3)
    B, page, width, num, V = 6, 16, 6, 64, 5000
    g = torch.Generator(device=DEV).manual_seed(3)
    k, v = (torch.randn((2, num, page, 2, 16), generator=g, device=DEV).to(BF16) for _ in range(2))
    a, b = _empty_set(B, width, num), _empty_set(B, width, num)
    cache = ptd.KVCache(k, v, 2, 16, page, a.block_table)
    ws, status = _fork_space(cache, a, b), torch.zeros(1, **I32)
    parents, lens = torch.zeros(B, **I32), torch.zeros(B, **I32)
    same, back = torch.arange(B, **I32), torch.zeros(B, **I32)
    logits, tokens = torch.zeros((B, V), dtype=BF16, device=DEV), torch.zeros(B, **I32)
    out = [torch.zeros(B, device=DEV), torch.zeros(B, device=DEV), torch.zeros((B, 3), **I32), torch.zeros((B, 3), device=DEV)]
    hidden, head = torch.zeros((B, 64), dtype=BF16, device=DEV), torch.randn((V, 64), generator=g, device=DEV).to(BF16)
    out2 = [torch.zeros_like(x) for x in out]
    ws2 = torch.empty(ptd.lm_head_logprobs_workspace_size(B, V, 3), dtype=torch.uint8, device=DEV)

    def step():
        ptd.page_fork(cache, a, b, parents, lens, ws, status)
        back.copy_(lens)
        ptd.page_fork(cache, b, a, same, back, ws, status)
        ptd.token_logprobs(logits, tokens, *out, status)
        ptd.lm_head_logprobs(hidden, head, tokens, *out2, ws2, status)

    graphs = []
    for _ in range(2):
        gr = torch.cuda.CUDAGraph()
        with torch.cuda.graph(gr):
            step()
        graphs.append(gr)
    table = [[i * 5 + j for j in range(5)] for i in range(B)]
    length = [int(rng.integers(1, 5 * page + 1)) for _ in range(B)]
    table = [t[:-(-n // page)] for t, n in zip(table, length)]
    free = [x for x in range(num) if not any(x in t for t in table)]
    a.block_table.copy_(torch.tensor([t + [-1] * (width - len(t)) for t in table], **I32))
    a.held.copy_(torch.tensor([len(t) for t in table], **I32))
    a.free_pages[:len(free)] = torch.tensor(free, **I32)
    a.free_count.fill_(len(free))
    content = [[k[:, t[i // page], i % page].clone() for i in range(n)] for t, n in zip(table, length)]
    for i in range(6):
        p = [int(rng.integers(0, B)) for _ in range(B)]
        n = [int(rng.integers(1, length[x] + 1)) if rng.random() < 0.5 else length[x] for x in p]
        parents.copy_(torch.tensor(p, **I32))
        lens.copy_(torch.tensor(n, **I32))
        logits.copy_((3 * torch.randn((B, V), generator=g, device=DEV)).to(BF16))
        hidden.copy_(torch.randn((B, 64), generator=g, device=DEV).to(BF16))
        tokens.copy_(torch.randint(0, V, (B,), generator=g, device=DEV))
        graphs[i % 2].replay()
        torch.cuda.synchronize()
        assert int(status) == 0
        content, length = [content[x][:m] for x, m in zip(p, n)], n
        t = a.block_table.tolist()
        for x in range(B):
            for j, want in enumerate(content[x]):
                assert torch.equal(k[:, t[x][j // page], j % page], want)
        assert int(a.free_count) == num - len({y for r, h in zip(t, a.held.tolist()) for y in r[:h]})
        for o, z, tol in ((out, logits.double(), 2.0 ** -16), (out2, hidden.double() @ head.double().t(), 2.0 ** -12)):
            exact = torch.log_softmax(z, -1)
            assert ((o[0].double() - exact.gather(1, tokens.long()[:, None])[:, 0]).abs() <= tol).all()
            assert ((o[3].double() - exact.topk(3).values).abs() <= tol).all()


def test_calls_on_streams_of_their_own():
    g = torch.Generator(device=DEV).manual_seed(4)
    xs = []
    for i in range(3):
        logits = torch.randn((70 + i, 40000 + 8 * i), generator=g, device=DEV).to(BF16)
        h, w = (torch.randn(s, generator=g, device=DEV).to(BF16) for s in ((150 + i, 256), (3000 + i, 256)))
        n = logits.shape[0]
        out = [torch.zeros(n, device=DEV), torch.zeros(n, device=DEV), torch.zeros((n, 4), **I32), torch.zeros((n, 4), device=DEV)]
        m = h.shape[0]
        out2 = [torch.zeros(m, device=DEV), torch.zeros(m, device=DEV), torch.zeros((m, 4), **I32), torch.zeros((m, 4), device=DEV)]
        ws = torch.empty(ptd.lm_head_logprobs_workspace_size(m, w.shape[0], 4), dtype=torch.uint8, device=DEV)
        xs.append((logits, torch.zeros(n, **I32), out, h, w, torch.ones(m, **I32), out2, ws, torch.zeros(1, **I32), torch.cuda.Stream()))
    torch.cuda.synchronize()
    for _ in range(6):
        for logits, t, out, h, w, t2, out2, ws, status, s in xs:
            ptd.token_logprobs(logits, t, *out, status, 0.9, stream=s)
            ptd.lm_head_logprobs(h, w, t2, *out2, ws, status, 0.9, stream=s)
    torch.cuda.synchronize()
    for logits, t, out, h, w, t2, out2, ws, status, s in xs:
        assert int(status) == 0
        for z, o, tok, tol in ((logits.double(), out, t, 2.0 ** -16), (h.double() @ w.double().t(), out2, t2, 2.0 ** -10)):
            p = torch.log_softmax(z / 0.9, -1)
            assert ((o[0].double() - p.gather(1, tok.long()[:, None])[:, 0]).abs() <= tol).all()
            assert ((o[3].double() - p.topk(4).values).abs() <= tol).all()


def test_offsets_past_32_bits():
    """Rows, layers and pages whose elements are 2^31 and more in."""
    g = torch.Generator(device=DEV).manual_seed(6)
    rows, stride, vocab = 5, 1 << 29, 4000
    flat = torch.zeros((rows - 1) * stride + vocab, dtype=BF16, device=DEV)
    logits = flat.as_strided((rows, vocab), (stride, 1))
    logits.copy_(torch.randn((rows, vocab), generator=g, device=DEV).to(BF16))
    out = [torch.zeros(rows, device=DEV), torch.zeros(rows, device=DEV), torch.zeros((rows, 2), **I32), torch.zeros((rows, 2), device=DEV)]
    t, status = torch.full((rows,), 3, **I32), torch.zeros(1, **I32)
    ptd.token_logprobs(logits, t, *out, status)
    p = torch.log_softmax(logits.double(), -1)
    assert ((out[0].double() - p[:, 3]).abs() <= 2.0 ** -16).all() and ((out[3].double() - p.topk(2).values).abs() <= 2.0 ** -16).all()
    # hidden states and weights as far apart
    d = 64
    wide = torch.zeros(3 * stride + d, dtype=BF16, device=DEV)
    h = wide.as_strided((4, d), (stride, 1))
    h.copy_(torch.randn((4, d), generator=g, device=DEV).to(BF16))
    w = flat.as_strided((4, d), (stride, 1))
    w.copy_(torch.randn((4, d), generator=g, device=DEV).to(BF16))
    out = [torch.zeros(4, device=DEV), None, torch.zeros((4, 2), **I32), torch.zeros((4, 2), device=DEV)]
    ws = torch.empty(ptd.lm_head_logprobs_workspace_size(4, 4, 2), dtype=torch.uint8, device=DEV)
    ptd.lm_head_logprobs(h, w, torch.full((4,), 3, **I32), *out, ws, status)
    p = torch.log_softmax(h.double() @ w.double().t(), -1)
    assert ((out[0].double() - p[:, 3]).abs() <= 2.0 ** -14).all() and ((out[3].double() - p.topk(2).values).abs() <= 2.0 ** -14).all()
    del flat, wide, logits, h, w
    torch.cuda.empty_cache()
    # a cache of 2^31 elements and more a layer
    page, hkv, dim = 128, 8, 128
    num = (1 << 31) // (page * hkv * dim) + 3
    k, v = (torch.zeros((2, num, page, hkv, dim), dtype=BF16, device=DEV) for _ in range(2))
    far = num - 1
    k[:, far] = torch.randn((2, page, hkv, dim), generator=g, device=DEV).to(BF16)
    v[:, far] = torch.randn((2, page, hkv, dim), generator=g, device=DEV).to(BF16)
    a, b = _empty_set(1, 4, num), _empty_set(2, 4, num)
    a.block_table[0, 0] = far
    a.held.fill_(1)
    a.free_pages[:2] = torch.tensor([5, far - 1], **I32)
    a.free_count.fill_(2)
    cache = ptd.KVCache(k, v, hkv, dim, page, a.block_table)
    ptd.page_fork(cache, a, b, torch.zeros(2, **I32), torch.tensor([100, 77], **I32), _fork_space(cache, a, b), status)
    assert b.block_table[:, 0].tolist() == [far, far - 1] and int(b.free_count) == 1
    for x in (k, v):
        assert torch.equal(x[:, far - 1, :77], x[:, far, :77]) and (x[:, far - 1, 77:] == 0).all() and (x[:, far, :100] != 0).any()
    q = torch.randn((1, hkv, dim), generator=g, device=DEV).to(BF16)
    kn, vn, w, out = q.flip(1).contiguous(), q.flip(2).contiguous(), torch.ones(dim, dtype=BF16, device=DEV), torch.empty_like(q)
    cache = ptd.KVCache(k, v, hkv, dim, page, b.block_table[:1].contiguous())
    slot = far * page + 101
    prompt = ptd.Prompt(torch.tensor([0, 1], **I32), torch.tensor([101], **I32), 1, 1, 101)
    ptd.prompt_norm_rope_append(prompt, cache, 1, torch.tensor([slot], **I32), torch.tensor([101], **I32), q, kn, vn, out, w, w, 1e-6,
                                1e4, status)
    assert torch.equal(v[1, far, 101], vn[0]) and (v[0, far, 101] != vn[0]).any()
    want = _normed(kn, w, [101], 1e4, 1e-6)
    assert ((k[1, far, 101].double() - want[0]).abs() <= want[0].abs() * 2.0 ** -8 * 1.01 + 2.0 ** -16).all()
    k[1, far, 101], v[1, far, 101] = 0, 0
    tree = ptd.Tree(torch.tensor([0, 1], **I32), torch.tensor([-1], **I32), torch.tensor([101], **I32), 1, 101)
    ptd.tree_norm_rope_append(tree, cache, 1, q[None], kn[None], vn[None], out[None], w[None], w[None], 1e-6, 1e4, status)
    assert torch.equal(v[1, far, 101], vn[0]) and ((k[1, far, 101].double() - want[0]).abs() <= want[0].abs() * 2.0 ** -8 * 1.01 + 2.0 ** -16).all()
    assert int(status) == 0


def _one_of_each():
    g = torch.Generator(device=DEV).manual_seed(8)
    hq, hkv, d, page, n = 4, 2, 128, 16, 9
    k, v = (torch.zeros((2, 10, page, hkv, d), dtype=BF16, device=DEV) for _ in range(2))
    a, b = _empty_set(1, 3, 10), _empty_set(2, 3, 10)
    a.block_table[0, :2] = torch.tensor([4, 7], **I32)
    a.held.fill_(2)
    a.free_pages[:3] = torch.tensor([1, 2, 3], **I32)
    a.free_count.fill_(3)
    k.copy_(torch.randn(k.shape, generator=g, device=DEV))
    cache, status = ptd.KVCache(k, v, hkv, d, page, a.block_table), torch.zeros(1, **I32)
    launches = [ptd.page_fork(cache, a, b, torch.zeros(2, **I32), torch.tensor([20, 20], **I32), _fork_space(cache, a, b), status)]
    q, kn, vn = (torch.randn((n, h, d), generator=g, device=DEV).to(BF16) for h in (hq, hkv, hkv))
    w = torch.randn((2, d), generator=g, device=DEV).to(BF16)
    prompt = ptd.Prompt(torch.tensor([0, n], **I32), torch.tensor([20], **I32), n, n, 20)
    slots, pos = torch.arange(70, 70 + n, **I32), torch.arange(20, 20 + n, **I32)
    out, out2 = torch.zeros_like(q), torch.zeros((1, n, hq, d), dtype=BF16, device=DEV)
    launches.append(ptd.prompt_norm_rope_append(prompt, cache, 1, slots, pos, q, kn, vn, out, w[0], w[1], 1e-6, 1e4, status))
    tree = ptd.Tree(torch.tensor([0, n], **I32), torch.arange(-1, n - 1, **I32), torch.tensor([20], **I32), n, 20)
    where = torch.zeros(n, **I32)
    launches.append(ptd.tree_norm_rope_append(tree, cache, 0, q[None], kn[None], vn[None], out2, w[:1], w[1:], 1e-6, 1e4, status, where))
    res = [k, v, b.block_table, b.held, b.free_pages, b.free_count, out, out2, where]
    logits, tokens = torch.randn((n, 3000), generator=g, device=DEV)[:, 3:], torch.arange(n, **I32)
    h, head = (torch.randn(s, generator=g, device=DEV).to(BF16) for s in ((n, 128), (500, 128)))
    ws = torch.empty(ptd.lm_head_logprobs_workspace_size(n, 500, 5), dtype=torch.uint8, device=DEV)
    for kk in (5, 0):
        o = [[torch.zeros(n, device=DEV), torch.zeros(n, device=DEV) if kk else None] +
             ([torch.zeros((n, kk), **I32), torch.zeros((n, kk), device=DEV)] if kk else [None, None]) for _ in range(2)]
        launches.append(ptd.token_logprobs(logits, tokens, *o[0], status, 0.8))
        launches.append(ptd.lm_head_logprobs(h, head, tokens, *o[1], ws, status, 0.8))
        res += [x for y in o for x in y if x is not None]
    torch.cuda.synchronize()
    assert int(status) == 0
    return launches, res


def test_native_and_ctypes_paths_agree(monkeypatch):
    calls, taken = ptd._native(), {}

    class Record:
        def __getattr__(self, name):
            def call(*a):
                taken.setdefault(name, []).append(getattr(calls, name)(*a))
                return taken[name][-1]

            return call

    class Refuse:
        def __getattr__(self, name):
            return lambda *a: None

    monkeypatch.setattr(ptd, "_calls", Record())
    native = _one_of_each()
    assert {n: len(r) for n, r in taken.items()} == {"page_fork": 1, "prompt_norm_rope_append": 1, "tree_norm_rope_append": 1,
                                                     "token_logprobs": 2, "lm_head_logprobs": 2}
    assert all(isinstance(x, int) and x > 0 for r in taken.values() for x in r), taken
    monkeypatch.setattr(ptd, "_calls", Refuse())
    plain = _one_of_each()
    assert native[0] == plain[0] == [2, 1, 1, 1, 2, 1, 2]
    for i, (a, b) in enumerate(zip(native[1], plain[1])):
        assert torch.equal(a, b), i


def test_binding_refuses_wrong_tensors():
    x, t = torch.randn((4, 100), device=DEV), torch.zeros(4, **I32)
    lp, st = torch.zeros(4, device=DEV), torch.zeros(1, **I32)
    idx, val = torch.zeros((4, 2), **I32), torch.zeros((4, 2), device=DEV)
    call = lambda logits=x, tokens=t, l=lp, e=None, i=idx, v=val, s=st, T=1.0: ptd.token_logprobs(logits, tokens, l, e, i, v, s, T)
    for err, kw in ((TypeError, dict(logits=x.half())), (ValueError, dict(logits=x.cpu())), (ValueError, dict(logits=x[:, ::2])),
                    (ValueError, dict(tokens=t[:3])), (TypeError, dict(tokens=t.long())), (ValueError, dict(l=lp[:2])),
                    (TypeError, dict(l=lp.double())), (ValueError, dict(e=lp[:3])), (ValueError, dict(i=None)), (ValueError, dict(v=None)),
                    (ValueError, dict(v=val[:, :1])), (ValueError, dict(i=idx[:2], v=val[:2])), (TypeError, dict(i=idx.long())),
                    (TypeError, dict(s=st.float())), (ptd.PtdError, dict(T=0.0)), (ptd.PtdError, dict(l=x[0, :4]))):
        with pytest.raises(err):
            call(**kw)
    wide = torch.zeros((4, 17), **I32), torch.zeros((4, 17), device=DEV)
    with pytest.raises(ptd.PtdError):
        call(i=wide[0], v=wide[1])
    h, w = torch.zeros((4, 64), dtype=BF16, device=DEV), torch.zeros((100, 64), dtype=BF16, device=DEV)
    ws = torch.empty(ptd.lm_head_logprobs_workspace_size(4, 100, 2), dtype=torch.uint8, device=DEV)
    call = lambda hidden=h, weight=w, tokens=t, work=ws: ptd.lm_head_logprobs(hidden, weight, tokens, lp, None, idx, val, work, st)
    for err, kw in ((TypeError, dict(hidden=h.float())), (ValueError, dict(weight=w[:, :32])), (ValueError, dict(tokens=t[:2])),
                    (ptd.PtdError, dict(work=ws[:64])), (ptd.PtdError, dict(hidden=h[:, :32], weight=w[:, :32]))):
        with pytest.raises(err):
            call(**kw)
    q, k = (torch.zeros((2, 5, n, 128), dtype=BF16, device=DEV) for n in (4, 2))
    cache = ptd.KVCache(torch.zeros((2, 1, 40, 2, 128), dtype=BF16, device=DEV), torch.zeros((2, 1, 40, 2, 128), dtype=BF16, device=DEV), 2, 128)
    tree = ptd.Tree(torch.tensor([0, 5], **I32), torch.arange(-1, 4, **I32), torch.tensor([7], **I32), 5, 7)
    wt = torch.ones((2, 128), dtype=BF16, device=DEV)
    call = lambda qq=q, kk=k, o=torch.zeros_like(q), a=wt, p=None, eps=1e-6: ptd.tree_norm_rope_append(
        tree, cache, 0, qq, kk, k.clone(), o, a, wt, eps, 1e4, st, p)
    for err, kw in ((TypeError, dict(qq=q.float())), (ValueError, dict(kk=q)), (ValueError, dict(o=q[:1])), (ValueError, dict(a=wt[0])),
                    (TypeError, dict(a=wt.float())), (ValueError, dict(p=torch.zeros(4, **I32))), (ptd.PtdError, dict(eps=-1.0)),
                    (ptd.PtdError, dict(o=k, qq=k.clone()))):   # q_out on k
        with pytest.raises(err):
            call(**kw)
    prompt = ptd.Prompt(torch.tensor([0, 5], **I32), torch.tensor([7], **I32), 5, 5, 7)
    sl = torch.arange(5, **I32)
    call = lambda a=wt[0], qq=q[0], s=sl: ptd.prompt_norm_rope_append(prompt, cache, 0, s, sl, qq, k[0], k[1], q[1], a, wt[1], 1e-6, 1e4, st)
    for err, kw in ((ValueError, dict(a=wt)), (TypeError, dict(a=wt[0].float())), (ValueError, dict(qq=q[0, :4])), (ValueError, dict(s=sl[:4]))):
        with pytest.raises(err):
            call(**kw)
    assert int(st) == 0 and (idx == 0).all() and (lp == 0).all()
