"""Operators around a step with several continuations, on the GPU against plain implementations in 64 bits: norms of the
heads with the rotary append (prompts and trees), log probabilities from logits and from hidden states, forks of pages,
and a run of them together.

Tolerances.  Norm and rotation: y = (x_j w_j c - x_i w_i s) n in fp32: n = (mean x^2 + eps)^(-1/2) has a relative error of at
most (D + 2) 2^-24 / 2 + 2^-24 (sums of D squares, their mean, the root), the weight's product, the factor and the two
products and one sum of the rotation 2^-24 each, the cosine and sine 2^-23 + p 2^-52: with M = |a| + |b| of the pair's normed
elements, M (D / 2 + 8) 2^-24, then half a step of the type (bf16: 2^-9 of a value's binade, 2^-8 |y| at most).
Log probabilities: with scores z = x / T, (z - max z) log2 e is off by 3 2^-24 of itself (difference, scale, product), so
by 3 1.45 2^-23 max|z| < 2^-21 max|z| / 0.9 and its part of a sum by that times ln 2; an exponential by 2^-22, a sum of n non-negative terms, added by threads of at most n / 256 + 8 each, by (n / 256 + 40) 2^-24 of
itself, logarithm and last products by 2^-22 of their values: the tolerance is 2^-21 max|z| + (n / 256 + 64) 2^-24 + 2^-21 |result|
(and for the entropy (n / 256 + 64) 2^-23 (1 + entropy) besides the first term: its two sums carry an error each)."""
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
NAN, INF = float("nan"), float("inf")


@pytest.fixture(scope="module", autouse=True)
def _built():
    import __graft_entry__

    __graft_entry__.build()


def _half_step(dtype):
    return torch.finfo(dtype).eps / 2


# ------------------------------------------------------------------ norms with the rotary append
def _norm_turn(x, w, pos, base, eps, dtype):
    """[n, h, D] normed and turned in 64 bits, and the tolerance of each element."""
    x, w, d = x.double().cpu().numpy(), w.double().cpu().numpy(), x.shape[-1]
    out = oracle.head_norm_rope(x, w, pos, float(base), eps)
    with np.errstate(all="ignore"):
        y = x * w / np.sqrt((x ** 2).mean(-1, keepdims=True) + eps)
    a, b = y[..., :d // 2], y[..., d // 2:]
    m = np.concatenate([np.abs(a) + np.abs(b)] * 2, -1)
    return out, m * ((d / 2 + 8) * 2.0 ** -24 + np.abs(np.asarray(pos, np.float64))[:, None, None] * 2.0 ** -50) \
        + np.abs(out) * _half_step(dtype) * 1.01 + 1e-30


def _same(got, want, tol, what):
    got = got.double().cpu().numpy()
    bad = ~((np.abs(got - want) <= tol) | (np.isnan(got) & np.isnan(want)))
    assert not bad.any(), (what, np.argwhere(bad)[:4].tolist(), got[bad][:4], want[bad][:4])


NORM_CASES = [(BF16, 32, 8, 128, 16, True), (BF16, 8, 8, 128, 0, False), (F32, 4, 2, 64, 32, True), (F32, 8, 1, 256, 0, True),
              (BF16, 3, 1, 96, 16, True), (F32, 2, 2, 12, 16, False), (BF16, 5, 5, 16, 0, True), (BF16, 2, 1, 256, 64, True),
              (F32, 6, 3, 8, 0, True)]


@pytest.mark.parametrize("tokens", [1, 7, 700])
@pytest.mark.parametrize("dtype,hq,hkv,d,page,fused", NORM_CASES)
def test_prompt_norm_rope_append(dtype, hq, hkv, d, page, fused, tokens):
    if (hkv * d * dtype.itemsize) % 16:
        pytest.skip("not a cache row")
    g = torch.Generator(device=DEV).manual_seed(tokens + d)
    rng = np.random.default_rng(tokens)
    pad, layers, rows = 3, 2, (tokens + 3 + 15) // 16 * 16 + 64
    n = tokens + pad
    shape = (layers, rows // page + 1, page, hkv, d) if page else (layers, 1, rows, hkv, d)
    table = torch.zeros((1, shape[1]), **I32) if page else None
    k = torch.full(shape, 5.0, dtype=dtype, device=DEV)
    v = torch.full(shape, 6.0, dtype=dtype, device=DEV)
    cache = ptd.KVCache(k, v, hkv, d, page, table)
    if fused:
        qkv = torch.randn((n, (hq + 2 * hkv) * d), generator=g, device=DEV).to(dtype)
        q, kn, vn = qkv[:, :hq * d].view(n, hq, d), qkv[:, hq * d:(hq + hkv) * d].view(n, hkv, d), qkv[:, -hkv * d:].view(n, hkv, d)
    else:
        q, kn, vn = (torch.randn((n, h, d), generator=g, device=DEV).to(dtype) for h in (hq, hkv, hkv))
    kn[0, 0] = 0   # a head of zeros stays one (eps > 0)
    wq, wk = ((1 + 0.3 * torch.randn(d, generator=g, device=DEV)).to(dtype) for _ in range(2))
    slots_h = np.concatenate([rng.permutation(rows)[:tokens], [-1] * pad]).astype(np.int32)
    pos_h = np.concatenate([rng.integers(0, 100000, tokens), [-1] * pad]).astype(np.int32)
    slots, pos = torch.tensor(slots_h, **I32), torch.tensor(pos_h, **I32)
    prompt = ptd.Prompt(torch.tensor([0, tokens], **I32), torch.zeros(1, **I32), n, tokens, 0)
    status = torch.zeros(1, **I32)
    out = torch.full((n, hq, d), 7.0, dtype=dtype, device=DEV)
    args = (prompt, cache, 1, slots, pos, q, kn, vn)
    assert ptd.prompt_norm_rope_append(*args, out, wq, wk, 1e-5, 10000.0, status) == 1
    first = [x.clone() for x in (out, k, v)]
    want, tol = _norm_turn(q[:tokens], wq, pos_h[:tokens], 10000.0, 1e-5, dtype)
    _same(out[:tokens], want, tol, "q")
    assert (out[tokens:] == 7.0).all()
    want, tol = _norm_turn(kn[:tokens], wk, pos_h[:tokens], 10000.0, 1e-5, dtype)
    at = torch.tensor(slots_h[:tokens], dtype=torch.long, device=DEV)
    _same(k[1].view(-1, hkv, d)[at], want, tol, "k")
    assert torch.equal(v[1].view(-1, hkv, d)[at], vn[:tokens])
    other = torch.ones(k[1].view(-1, hkv, d).shape[0], dtype=torch.bool, device=DEV)
    other[at] = False
    assert (k[0] == 5.0).all() and (v[0] == 6.0).all()
    assert (k[1].view(-1, hkv, d)[other] == 5.0).all() and (v[1].view(-1, hkv, d)[other] == 6.0).all()
    # in place, the same bits
    assert ptd.prompt_norm_rope_append(*args, q, wq, wk, 1e-5, 10000.0, status) == 1
    assert torch.equal(q[:tokens], first[0][:tokens]) and torch.equal(k, first[1]) and torch.equal(v, first[2])
    assert status.item() == 0


@pytest.mark.parametrize("dtype,hq,hkv,d,page,_", NORM_CASES)
@pytest.mark.parametrize("nodes,layers", [([1], 1), ([63], 5), ([7, 128, 1, 33], 2)])
def test_tree_norm_rope_append(dtype, hq, hkv, d, page, _, nodes, layers):
    if (hkv * d * dtype.itemsize) % 16:
        pytest.skip("not a cache row")
    g = torch.Generator(device=DEV).manual_seed(sum(nodes) + d)
    rng = np.random.default_rng(d)
    off = np.concatenate([[0], np.cumsum(nodes)])
    n, B, ctx = int(off[-1]), len(nodes), [17 * b + 5 for b in range(len(nodes))]
    parents = np.concatenate([[-1] + [int(rng.integers(0, i)) for i in range(1, t)] for t in nodes]).astype(np.int32)
    cap = max(c + t for c, t in zip(ctx, nodes)) + 2
    L = layers + 1
    if page:
        per = -(-cap // page)
        table_h = rng.permutation(B * per + 2)[:B * per].reshape(B, per).astype(np.int32)
        shape, table = (L, B * per + 2, page, hkv, d), torch.tensor(table_h, **I32)
    else:
        shape, table = (L, B, cap, hkv, d), None
    k, v = torch.full(shape, 5.0, dtype=dtype, device=DEV), torch.full(shape, 6.0, dtype=dtype, device=DEV)
    cache = ptd.KVCache(k, v, hkv, d, page, table)
    tree = ptd.Tree(torch.tensor(off, **I32), torch.tensor(parents, **I32), torch.tensor(ctx, **I32), max(nodes), max(ctx))
    q, kn, vn = (torch.randn((layers, n, h, d), generator=g, device=DEV).to(dtype) for h in (hq, hkv, hkv))
    wq, wk = ((1 + 0.3 * torch.randn((layers, d), generator=g, device=DEV)).to(dtype) for _ in range(2))
    out, status, where = torch.full_like(q, 7.0), torch.zeros(1, **I32), torch.zeros(n, **I32)
    assert ptd.tree_norm_rope_append(tree, cache, 1, q, kn, vn, out, wq, wk, 1e-6, 500000.0, status, where) == 1
    pos, rows = [], []
    for b, t in enumerate(nodes):
        depth = []
        for i in range(t):
            depth.append(0 if i == 0 else depth[parents[off[b] + i]] + 1)
            slot = ctx[b] + i
            rows.append(int(table_h[b, slot // page]) * page + slot % page if page else b * cap + slot)
        pos += [ctx[b] + x for x in depth]
    assert where.tolist() == pos and status.item() == 0
    at = torch.tensor(rows, device=DEV)
    other = torch.ones(k[1].view(-1, hkv, d).shape[0], dtype=torch.bool, device=DEV)
    other[at] = False
    for l in range(layers):
        want, tol = _norm_turn(q[l], wq[l], pos, 500000.0, 1e-6, dtype)
        _same(out[l], want, tol, ("q", l))
        want, tol = _norm_turn(kn[l], wk[l], pos, 500000.0, 1e-6, dtype)
        _same(k[l + 1].view(-1, hkv, d)[at], want, tol, ("k", l))
        assert torch.equal(v[l + 1].view(-1, hkv, d)[at], vn[l])
        assert (k[l + 1].view(-1, hkv, d)[other] == 5.0).all()
    assert (k[0] == 5.0).all()
    first = k.clone()
    ptd.tree_norm_rope_append(tree, cache, 1, q, kn, vn, q, wq, wk, 1e-6, 500000.0, status)   # in place, the same bits
    assert torch.equal(q, out) and torch.equal(k, first)


def test_norms_of_hard_rows():
    """Zeros without eps, infinities and NaN stay in their own heads; tiny and large values keep their precision."""
    d, hq = 128, 4
    q = torch.randn((2, hq, d), device=DEV)
    q[0, 0], q[0, 1, 5], q[0, 2, 9] = 0.0, INF, NAN
    q[1, 0] *= 1e-12
    q[1, 1] *= 1e15
    k = torch.randn((2, hq, d), device=DEV)
    cache = ptd.KVCache(torch.zeros((1, 1, 4, hq, d), device=DEV), torch.zeros((1, 1, 4, hq, d), device=DEV), hq, d)
    prompt = ptd.Prompt(torch.tensor([0, 2], **I32), torch.zeros(1, **I32), 2, 2, 0)
    slots, pos, status = torch.tensor([2, 0], **I32), torch.tensor([3, 1 << 20], **I32), torch.zeros(1, **I32)
    w, out = torch.rand(d, device=DEV), torch.zeros((2, hq, d), device=DEV)
    ptd.prompt_norm_rope_append(prompt, cache, 0, slots, pos, q, k, k.clone(), out, w, w, 0.0, 10000.0, status)
    assert out[0, 0].isnan().all() and out[0, 2].isnan().all() and out[0, 1].isnan().any()
    want, tol = _norm_turn(q[1:], w, [1 << 20], 10000.0, 0.0, F32)
    _same(out[1:], want, tol, "q")
    _same(out[:1, 3:], *_norm_turn(q[:1, 3:], w, [3], 10000.0, 0.0, F32), "q")


def test_norm_append_reports_slots_outside_the_cache():
    d, n = 128, 5
    cache = ptd.KVCache(torch.zeros((1, 1, 4, 1, d), dtype=BF16, device=DEV), torch.zeros((1, 1, 4, 1, d), dtype=BF16, device=DEV), 1, d)
    prompt = ptd.Prompt(torch.tensor([0, n], **I32), torch.zeros(1, **I32), n, n, 0)
    slots, pos, status = torch.tensor([0, 4, -2, 1 << 30, 3], **I32), torch.arange(n, **I32), torch.zeros(1, **I32)
    q = torch.randn((n, 2, d), device=DEV).to(BF16)
    k = torch.randn((n, 1, d), device=DEV).to(BF16)
    w, out = torch.ones(d, dtype=BF16, device=DEV), torch.full((n, 2, d), 7.0, dtype=BF16, device=DEV)
    ptd.prompt_norm_rope_append(prompt, cache, 0, slots, pos, q, k, k.clone(), out, w, w, 1e-6, 10000.0, status)
    assert status.item() == ptd.INVALID_BATCH
    assert (out[1:4] == 7.0).all() and (out[0] != 7.0).any() and (out[4] != 7.0).any()
    assert (cache.k[0, 0, 1:3] == 0).all() and (cache.k[0, 0, 3] != 0).any()


# ------------------------------------------------------------------ log probabilities
def _check_logprobs(logits, tokens, T, k, logprob, entropy, idx, val, accurate=0.0):
    """Against 64 bits; accurate: the largest error of a logit."""
    x = logits.double().cpu()
    z = x / T
    n = x.shape[1]
    p = torch.log_softmax(z, -1)
    dead = (x == -INF).all(-1)
    p[dead] = -INF
    finite = torch.where(z.isfinite(), z.abs(), 0.0).amax(-1)
    base = (finite * 2.0 ** -21 + (n / 256 + 64) * 2.0 ** -24 + 2 * accurate / T)
    t = tokens.cpu().long()
    inside = (t >= 0) & (t < n)
    want = torch.where(inside, p.gather(1, t.clamp(0, n - 1)[:, None])[:, 0], -INF)

    def close(got, want, tol):
        got = got.double().cpu()
        ok = ((got - want).abs() <= tol) | (got == want) | (got.isnan() & want.isnan())
        assert ok.all(), (got[~ok][:4], want[~ok][:4], tol.expand_as(want)[~ok][:4])

    close(logprob, want, base + want.abs().nan_to_num(0, 0, 0) * 2.0 ** -21)
    if entropy is not None:
        e = -(p.exp() * p.masked_fill(p == -INF, 0.0)).sum(-1)
        close(entropy, e, (base + (n / 256 + 64) * 2.0 ** -23) * (1 + e.abs()) + e.abs() * 2 * accurate / T)
    if k:
        clean = ~x.isnan().any(-1)
        order = torch.sort(torch.where(x == 0, 0.0, x), dim=-1, descending=True, stable=True).indices[:, :k]
        if accurate == 0:
            assert torch.equal(idx.cpu().long()[clean], order[clean])
        got = idx.cpu().long()[clean]
        assert all(len(set(r.tolist())) == k for r in got)
        top = p[clean].gather(1, got)
        close(val[clean.to(DEV)], top, base[clean, None] + top.abs().nan_to_num(0, 0, 0) * 2.0 ** -21)


def _outputs(rows, k):
    return (torch.full((rows,), 7.0, device=DEV), torch.full((rows,), 7.0, device=DEV),
            torch.full((rows, k), 7, **I32) if k else None, torch.full((rows, k), 7.0, device=DEV) if k else None)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("rows,vocab,k,T", [(1, 1, 1, 1.0), (3, 5, 5, 1.0), (2, 17, 16, 0.5), (1, 128256, 8, 1.0), (63, 32000, 4, 0.7),
                                            (300, 50257, 1, 1.3), (2000, 1000, 16, 1.0), (5, 262144, 0, 1.0), (9, 16391, 2, 3.0),
                                            (700, 65541, 3, 1.0)])
def test_token_logprobs(dtype, rows, vocab, k, T):
    g = torch.Generator(device=DEV).manual_seed(vocab)
    logits = (3 * torch.randn((rows, vocab), generator=g, device=DEV)).to(dtype)
    logits[0, vocab // 2] = 20.0
    tokens = torch.randint(-1, vocab + 1, (rows,), generator=g, device=DEV).to(torch.int32)
    tokens[0] = vocab // 2
    out, status = _outputs(rows, k), torch.zeros(1, **I32)
    assert ptd.token_logprobs(logits, tokens, *out, status, T) == 1
    assert status.item() == 0
    _check_logprobs(logits, tokens, T, k, *out)
    again = _outputs(rows, k)
    ptd.token_logprobs(logits, tokens, again[0], None, again[2], again[3], status, T)   # no entropy; the same bits
    assert torch.equal(again[0], out[0]) and (again[1] == 7.0).all()
    if k:
        assert torch.equal(again[2], out[2]) and torch.equal(again[3], out[3])


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("rows,vocab,shift,extra", [(5, 1000, 1, 7), (4, 70001, 3, 2), (17, 513, 5, 0)])
def test_token_logprobs_of_rows_off_16_bytes(dtype, rows, vocab, shift, extra):
    g = torch.Generator(device=DEV).manual_seed(vocab)
    wide = torch.full((rows * (vocab + extra) + shift,), 99.0, dtype=dtype, device=DEV)
    logits = wide[shift:].as_strided((rows, vocab), (vocab + extra, 1), shift)
    logits.copy_((3 * torch.randn((rows, vocab), generator=g, device=DEV)).to(dtype))
    tokens = torch.randint(0, vocab, (rows,), generator=g, device=DEV).to(torch.int32)
    out, status = _outputs(rows, 6), torch.zeros(1, **I32)
    ptd.token_logprobs(logits, tokens, *out, status)
    _check_logprobs(logits, tokens, 1.0, 6, *out)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("vocab", [40, 5000, 128256])
def test_token_logprobs_of_masked_and_broken_rows(dtype, vocab):
    g = torch.Generator(device=DEV).manual_seed(vocab)
    x = torch.randn((12, vocab), generator=g, device=DEV)
    lowest = torch.finfo(dtype).min
    x[0] = -INF                                    # nothing left
    x[1] = -INF
    x[1, vocab - 1] = -3.0                         # one token left
    x[2, 7:] = -INF
    x[3] = lowest                                  # a mask of the type's lowest value, everywhere
    x[4, 3:] = lowest
    x[5, 11] = NAN
    x[6, 13] = INF
    x[7] = 0.25                                    # all equal: the lowest indices
    x[8, ::2] = 0.0
    x[8, 1::2] = -0.0                              # signed zeros are equal
    x[9] = NAN
    x[10] = -1e30
    x[10, 5] = 1e30                                # one certain token
    x[11, :] = torch.linspace(-30, 30, vocab, device=DEV)
    logits = x.to(dtype)
    tokens = torch.tensor([3, vocab - 1, 2, 9, 1, 2, 13, 4, 5, 6, 5, vocab - 2], **I32)
    out, status = _outputs(12, 16), torch.zeros(1, **I32)
    ptd.token_logprobs(logits, tokens, *out, status)
    lp, e = out[0].cpu(), out[1].cpu()
    assert lp[0] == -INF and e[0] == 0 and (out[3][0] == -INF).all() and out[2][0].tolist() == list(range(16))
    assert lp[1] == 0 and e[1] == 0 and out[2][1, 0] == vocab - 1 and (out[3][1, 1:] == -INF).all()
    for r in (5, 6, 9):
        assert lp[r].isnan() and e[r].isnan() and out[3][r].isnan().all()
    if vocab == 40:
        want = oracle.token_logprobs(logits.double().cpu().numpy()[[0, 1, 2, 7, 8, 11]], tokens.cpu().numpy()[[0, 1, 2, 7, 8, 11]], 1.0, 16)
        for got, w in zip(out, want):
            got = got.double().cpu().numpy()[[0, 1, 2, 7, 8, 11]]
            with np.errstate(invalid="ignore"):   # -inf - -inf
                assert ((got == w) | (np.abs(got - w) <= 2.0 ** -16)).all()
    good = [r for r in range(12) if r not in (0, 5, 6, 9)]
    sel = torch.tensor(good, device=DEV)
    _check_logprobs(logits[sel], tokens[sel], 1.0, 16, *(o[sel] for o in out))
    assert status.item() == 0


def _lm_case(rows, vocab, d, seed, dtype=BF16):
    """Grids whose products' sums are exact in 32 bits, in any order."""
    g = torch.Generator(device=DEV).manual_seed(seed)
    unit = 2.0 ** -round(math.log2(math.sqrt(d)))
    grid = lambda s: (torch.randn(s, generator=g, device=DEV) * 8).round() / 8
    return grid((rows, d)).to(dtype), (grid((vocab, d)) * 2 * unit).to(dtype), \
        torch.randint(-1, vocab + 1, (rows,), generator=g, device=DEV).to(torch.int32)


@pytest.mark.parametrize("rows,vocab,d,k,T", [(1, 1, 64, 1, 1.0), (1, 5, 64, 5, 1.0), (63, 128256, 256, 8, 0.7), (128, 1000, 512, 16, 1.0),
                                              (129, 1000, 512, 4, 1.0), (300, 257, 128, 3, 2.0), (1500, 4097, 192, 0, 1.0),
                                              (1025, 32000, 64, 1, 1.0), (2500, 300, 64, 16, 1.0), (257, 50257, 448, 2, 1.0),
                                              (1200, 130, 64, 8, 1.0), (3000, 20000, 128, 5, 1.0)])
def test_lm_head_logprobs(rows, vocab, d, k, T):
    h, w, tokens = _lm_case(rows, vocab, d, rows + vocab)
    out, status = _outputs(rows, k), torch.zeros(1, **I32)
    ws = torch.full((ptd.lm_head_logprobs_workspace_size(rows, vocab, k),), 255, dtype=torch.uint8, device=DEV)
    assert ptd.lm_head_logprobs(h, w, tokens, *out, ws, status, T) == 2
    assert status.item() == 0
    for r0 in range(0, rows, 512):
        r = slice(r0, r0 + 512)
        logits = h[r].double() @ w.double().t()
        _check_logprobs(logits, tokens[r], T, k, *(o[r] if o is not None else None for o in out))
    again = _outputs(rows, k)
    ptd.lm_head_logprobs(h, w, tokens, *again, ws, status, T)
    assert all(torch.equal(a, b) for a, b in zip(again, out) if a is not None)


def test_lm_head_logprobs_of_strided_rows_and_real_values():
    """Random values: a logit is off by d 2^-24 sum |h w| at most, as it accumulates in 32 bits (twice that where it truncates)."""
    rows, vocab, d = 200, 3001, 1024
    g = torch.Generator(device=DEV).manual_seed(1)
    h = torch.randn((rows, d + 8), generator=g, device=DEV).to(BF16)[:, 8:]
    w = (torch.randn((vocab, 2 * d), generator=g, device=DEV) / 16).to(BF16)[:, :d]
    tokens = torch.randint(0, vocab, (rows,), generator=g, device=DEV).to(torch.int32)
    out, status = _outputs(rows, 4), torch.zeros(1, **I32)
    ws = torch.empty(ptd.lm_head_logprobs_workspace_size(rows, vocab, 4), dtype=torch.uint8, device=DEV)
    ptd.lm_head_logprobs(h, w, tokens, *out, ws, status, 1.5)
    size = float((h.double().abs() @ w.double().abs().t()).max())
    _check_logprobs(h.double() @ w.double().t(), tokens, 1.5, 4, *out, accurate=d * 2.0 ** -23 * size)
    assert status.item() == 0


def test_lm_head_logprobs_of_broken_rows():
    rows, vocab, d = 140, 700, 64
    h, w, tokens = _lm_case(rows, vocab, d, 3)
    tokens.clamp_(0, vocab - 1)
    h[5, 3], h[130, 0] = NAN, INF
    out, status = _outputs(rows, 4), torch.zeros(1, **I32)
    ws = torch.empty(ptd.lm_head_logprobs_workspace_size(rows, vocab, 4), dtype=torch.uint8, device=DEV)
    ptd.lm_head_logprobs(h, w, tokens, *out, ws, status)
    for r in (5, 130):
        assert out[0][r].isnan() and out[1][r].isnan() and out[3][r].isnan().all()
    good = torch.tensor([r for r in range(rows) if r not in (5, 130)], device=DEV)
    _check_logprobs(h[good].double() @ w.double().t(), tokens[good], 1.0, 4, *(o[good] for o in out))


# ------------------------------------------------------------------ forks
class Pages:
    """A random paged state: sequences that share prefixes, a stack of free pages, K and V of random values."""

    def __init__(self, seed, B, to, P, longest, layers=2, hkv=2, d=16, dtype=BF16, spare=None):
        rng = np.random.default_rng(seed)
        table, at = [], 0
        for b in range(B):
            own = int(rng.integers(0, longest + 1))
            shared = list(table[int(rng.integers(0, b))]) if b and rng.random() < 0.5 else []
            shared = shared[:int(rng.integers(0, len(shared) + 1))]
            own = max(0, own - len(shared))
            table.append(shared + list(range(at, at + own)))
            at += own
        spare = to + 2 if spare is None else spare
        self.num_pages = max(at + spare, 1)
        perm = rng.permutation(self.num_pages)
        self.table = [[int(perm[x]) for x in r] for r in table]
        self.held = [len(r) for r in table]
        self.free = [int(x) for x in perm[at:]][:max(0, self.num_pages - at)]
        self.P, self.W, self.B, self.to = P, longest + 1, B, to
        self.parents = [int(rng.integers(-1, B)) for _ in range(to)]
        self.lens = [int(rng.integers(0, self.held[p] * P + 1)) if p >= 0 else int(rng.integers(-5, 5)) for p in self.parents]
        g = torch.Generator(device=DEV).manual_seed(seed)
        shape = (layers, self.num_pages, P, hkv, d)
        self.k, self.v = (torch.randn(shape, generator=g, device=DEV).to(dtype) for _ in range(2))
        t = np.full((B, self.W), -7, np.int32)
        for b, r in enumerate(self.table):
            t[b, :len(r)] = r
        f = np.full(self.num_pages, -8, np.int32)
        f[:len(self.free)] = self.free
        self.source = ptd.PageSet(torch.tensor(t, **I32), torch.tensor(self.held, **I32), torch.tensor(f, **I32),
                                  torch.tensor([len(self.free)], **I32))
        self.target = ptd.PageSet(torch.full((to, self.W), -3, **I32), torch.full((to,), -3, **I32),
                                  torch.full((self.num_pages,), -3, **I32), torch.full((1,), -3, **I32))
        self.cache = ptd.KVCache(self.k, self.v, hkv, d, P, self.source.block_table)
        self.status = torch.zeros(1, **I32)

    def run(self, parents=None, lens=None):
        ws = torch.full((ptd.page_fork_workspace_size(self.cache, self.source, self.target),), 255, dtype=torch.uint8, device=DEV)
        p = torch.tensor(self.parents if parents is None else parents, **I32)
        n = torch.tensor(self.lens if lens is None else lens, **I32)
        return ptd.page_fork(self.cache, self.source, self.target, p, n, ws, self.status)

    def check(self, k0, v0):
        rows, stack, copies = oracle.page_fork(self.table, self.held, self.free, self.parents, self.lens, self.P)
        t = self.target
        got = t.block_table.cpu().tolist()
        assert t.held.tolist() == [len(r) for r in rows]
        for b, r in enumerate(rows):
            assert got[b] == r + [-3] * (self.W - len(r)), b
        assert t.free_count.tolist() == [len(stack)]
        assert t.free_pages.tolist() == stack + [-3] * (self.num_pages - len(stack))
        for x, y, n in copies:
            k0[:, y, :n], v0[:, y, :n] = k0[:, x, :n], v0[:, x, :n]
        assert torch.equal(self.k, k0) and torch.equal(self.v, v0)
        assert self.status.item() == 0


@pytest.mark.parametrize("seed,B,to,P,longest,kw", [
    (0, 1, 1, 16, 1, {}), (1, 1, 64, 16, 9, {}), (2, 8, 8, 32, 5, {}), (3, 40, 7, 64, 12, {}), (4, 7, 90, 128, 3, dict(layers=3)),
    (5, 300, 500, 16, 70, dict(layers=1, hkv=1, d=8)), (6, 1500, 900, 16, 40, dict(layers=1, hkv=1, d=8)),
    (7, 5, 6, 16, 4, dict(dtype=F32, hkv=3, d=4)), (8, 12, 12, 128, 6, dict(layers=2, hkv=8, d=128)), (9, 3, 3, 16, 0, {}),
    (10, 8192, 8192, 16, 2, dict(layers=1, hkv=1, d=8))])
def test_page_fork(seed, B, to, P, longest, kw):
    x = Pages(seed, B, to, P, longest, **kw)
    k0, v0 = x.k.clone(), x.v.clone()
    before = [t.clone() for t in (x.source.block_table, x.source.held, x.source.free_pages, x.source.free_count)]
    assert x.run() == 2
    x.check(k0, v0)
    assert x.run() == 2   # a call on the same state writes the same
    x.check(k0, v0)
    after = (x.source.block_table, x.source.held, x.source.free_pages, x.source.free_count)
    assert all(torch.equal(a, b) for a, b in zip(before, after))


def test_page_fork_shares_and_keeps():
    """By hand: four positions over a page; the first child keeps the partial page, one that has it whole takes it from all."""
    x = Pages(0, 2, 4, 16, 3, spare=5)
    x.table, x.held, x.W = [[4, 2, 6], [4, 1]], [3, 2], 4
    x.num_pages = x.num_pages if x.num_pages >= 9 else 9
    shape = (2, x.num_pages, 16, 2, 16)
    x.k, x.v = torch.randn(shape, device=DEV).to(BF16), torch.randn(shape, device=DEV).to(BF16)
    x.free = [0, 3, 5]
    x.source = ptd.PageSet(torch.tensor([[4, 2, 6, -1], [4, 1, -1, -1]], **I32), torch.tensor([3, 2], **I32),
                           torch.tensor([0, 3, 5] + [-1] * (x.num_pages - 3), **I32), torch.tensor([3], **I32))
    x.target = ptd.PageSet(torch.full((4, 4), -3, **I32), torch.zeros(4, **I32), torch.full((x.num_pages,), -3, **I32),
                           torch.zeros(1, **I32))
    x.cache = ptd.KVCache(x.k, x.v, 2, 16, 16, x.source.block_table)
    x.parents, x.lens = [1, 0, 0, 0], [20, 36, 36, 20]
    k0, v0 = x.k.clone(), x.v.clone()
    x.run()
    assert x.target.block_table.tolist() == [[4, 1, -3, -3], [4, 2, 6, -3], [4, 2, 5, -3], [4, 3, -3, -3]]
    assert x.target.free_pages[:1].tolist() == [0] and x.target.free_count.item() == 1
    x.check(k0, v0)


@pytest.mark.parametrize("what", ["held", "negative held", "parent", "parents", "len", "page", "free page", "count", "crowded"])
def test_page_fork_refused_as_a_whole(what):
    x = Pages(11, 6, 9, 16, 5)
    b = max(range(6), key=lambda i: x.held[i])
    parents, lens = [b] * 9, [x.held[b] * 16 - 3] * 9
    if what == "held":
        x.source.held[2] = x.W + 1
    elif what == "negative held":
        x.source.held[2] = -1
    elif what == "parent":
        parents[4] = 6
    elif what == "parents":
        parents[8] = -2
    elif what == "len":
        lens[3] = x.held[b] * 16 + 1
    elif what == "page":
        x.source.block_table[b, 0] = x.num_pages
    elif what == "free page":
        x.source.free_pages[0] = -1
    elif what == "count":
        x.source.free_count[0] = x.num_pages + 1
    else:
        x.source.free_count[0] = 3   # eight are needed
    k0, v0 = x.k.clone(), x.v.clone()
    x.run(parents, lens)
    assert x.status.item() == (ptd.NO_PAGES if what == "crowded" else ptd.INVALID_BATCH)
    assert (x.target.held == 0).all() and x.target.free_count.item() == 0
    assert (x.target.block_table == -3).all() and (x.target.free_pages == -3).all()
    assert torch.equal(x.k, k0) and torch.equal(x.v, v0)
