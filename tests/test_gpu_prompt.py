"""The prompt path on the GPU against the float64 oracle: pages, slots, rotary append, causal attention, and a run
of them together with the tree calls.

Tolerances of the attention, per output o = sum_j w_j v_j with S = sum_j w_j |v_j|: a weight rounded to bf16 is off
by 2^-8 of itself at most (bf16 caches), so S 2^-8; the output's rounding, |o| 2^-8 (fp32: 2^-24); a score q.k
accumulated over D products in fp32 is off by D 2^-23 sum |q k| at most (a truncating accumulator), its scaling
and the exponential by 2^-22 of the largest |score| + 2^-21, and a score's error e changes numerator and
denominator by e each: 2 e S; fp32 sums over n keys add n 2^-24 S to each of both."""
import decimal
import math
import threading

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


def _attention_tolerance(q, k, v, o, size, dtype, scale=None):
    n, hq, d = q.shape
    g = hq // k.shape[1]
    scale = 1 / math.sqrt(d) if scale is None else scale
    biggest = max(float((np.abs(q[:, h]) @ np.abs(k[:, h // g]).T).max()) for h in range(hq)) * scale
    e = d * 2.0 ** -23 * biggest + 2.0 ** -22 * biggest + 2.0 ** -21 + len(k) * 2.0 ** -24
    w, r = (2.0 ** -8, 2.0 ** -8) if dtype == BF16 else (0.0, 2.0 ** -24)
    return (w + 2 * e) * size * 1.01 + r * np.abs(o) + 1e-30


class Batch:
    """A cache full of NaN, but for the positions of `seqs` = [(context, new tokens)], and random q, k, v."""

    def __init__(self, seqs, hq, hkv, d=128, page=0, dtype=BF16, pad=0, layers=1, seed=0, spare=3, max_ctx=None,
                 max_tokens=None):
        self.ctx, self.new = [c for c, _ in seqs], [n for _, n in seqs]
        self.off = np.concatenate([[0], np.cumsum(self.new)]).astype(int)
        self.hq, self.hkv, self.d, self.page, self.dtype, self.layers = hq, hkv, d, page, dtype, layers
        B, self.N = len(seqs), int(self.off[-1]) + pad
        rng = np.random.default_rng(seed)
        longest = max(max(c + n for c, n in seqs), 1)
        if page:
            per = [-(-(c + n) // page) for c, n in seqs]
            self.num_pages = sum(per) + spare
            perm = rng.permutation(self.num_pages).astype(np.int32)
            table = np.full((B, max(max(per), 1) + 1), -1, np.int32)
            at = 0
            for b, n in enumerate(per):
                table[b, :n] = perm[at:at + n]
                at += n
            self.table_h = table
            self.table = torch.tensor(table, **I32)
            shape = (layers, self.num_pages, page, hkv, d)
        else:
            self.table, self.table_h = None, None
            shape = (layers, B, longest + spare, hkv, d)
        self.k = torch.full(shape, float("nan"), dtype=dtype, device=DEV)
        self.v = torch.full(shape, float("nan"), dtype=dtype, device=DEV)
        g = torch.Generator(device=DEV).manual_seed(seed)
        self.rows = []
        for b, (c, n) in enumerate(seqs):
            p = np.arange(c + n)
            r = table[b][p // page] * page + p % page if page else b * shape[2] + p
            self.rows.append(torch.tensor(r, dtype=torch.long, device=DEV))
            for l in range(layers):
                for x in (self.k, self.v):
                    x[l].view(-1, hkv, d)[self.rows[b]] = torch.randn((c + n, hkv, d), generator=g, device=DEV).to(dtype)
        self.q = torch.randn((self.N, hq, d), generator=g, device=DEV).to(dtype)
        self.out = torch.full((self.N, hq, d), 7.0, dtype=dtype, device=DEV)
        self.token_offsets, self.ctx_lens = torch.tensor(self.off, **I32), torch.tensor(self.ctx, **I32)
        self.status = torch.zeros(1, **I32)
        self.cache = ptd.KVCache(self.k, self.v, hkv, d, page, self.table)
        self.prompt = ptd.Prompt(self.token_offsets, self.ctx_lens, max(self.N, 1), max_tokens or max(max(self.new), 1),
                                 max(self.ctx) if max_ctx is None else max_ctx)

    def workspace(self):
        n = ptd.prompt_attention_workspace_size(self.prompt, self.cache, self.hq)
        return torch.full((n,), 255, dtype=torch.uint8, device=DEV) if n else None

    def attend(self, layer=0, q=None, workspace="own", **kw):
        ws = self.workspace() if workspace == "own" else workspace
        n = ptd.prompt_attention(self.prompt, self.cache, layer, self.q if q is None else q, self.out, self.status,
                                 workspace=ws, **kw)
        torch.cuda.synchronize()
        return n

    def kv(self, b, layer=0):
        return (x[layer].view(-1, self.hkv, self.d)[self.rows[b]].double().cpu().numpy() for x in (self.k, self.v))

    def check(self, layer=0, scale=None, seqs=None):
        out, q = self.out.double().cpu().numpy(), self.q.double().cpu().numpy()
        for b in range(len(self.new)) if seqs is None else seqs:
            if self.new[b] == 0:
                continue
            sl = slice(self.off[b], self.off[b + 1])
            k, v = self.kv(b, layer)
            o, size = oracle.causal_attention(q[sl], k, v, self.ctx[b], scale)
            tol = _attention_tolerance(q[sl], k, v, o, size, self.dtype, scale)
            bad = ~(np.abs(out[sl] - o) <= tol)
            assert not bad.any(), (b, np.argwhere(bad)[:4].tolist(), (np.abs(out[sl] - o) / tol).max())
        assert (out[self.off[-1]:] == 7.0).all()   # rows behind the last sequence


RAGGED = [(0, 1), (0, 130), (17, 64), (100, 0), (511, 33), (0, 0), (129, 1)]
CASES = {
    "one-token": dict(seqs=[(0, 1)], hq=8, hkv=8),
    "gqa-paged16-ragged": dict(seqs=RAGGED, hq=32, hkv=8, page=16, pad=5),
    "gqa-paged32": dict(seqs=[(31, 200), (64, 3)], hq=8, hkv=2, page=32),
    "gqa-paged64": dict(seqs=[(0, 257), (1, 63)], hq=16, hkv=2, page=64, pad=1),
    "gqa-paged128": dict(seqs=[(128, 128), (300, 5)], hq=8, hkv=2, page=128),
    "mha-contiguous": dict(seqs=[(0, 129), (0, 128), (127, 1), (1, 255)], hq=4, hkv=4),
    "group5": dict(seqs=[(3, 77), (0, 51), (200, 1)], hq=10, hkv=2),
    "group7-layer1": dict(seqs=[(0, 37), (90, 111)], hq=14, hkv=2, page=16, layers=2, layer=1),
    "group64": dict(seqs=[(0, 9), (140, 4)], hq=64, hkv=1),
    "group96": dict(seqs=[(5, 7)], hq=96, hkv=1),
    "group131": dict(seqs=[(5, 150)], hq=131, hkv=1),
    "group192": dict(seqs=[(120, 10)], hq=192, hkv=1),
    "long-split": dict(seqs=[(5000, 3)], hq=8, hkv=1, page=64),
    "long-split-contiguous": dict(seqs=[(2047, 2), (10, 1), (4000, 90)], hq=8, hkv=2),
    "bounds-above-lengths": dict(seqs=[(40, 30), (0, 2)], hq=8, hkv=2, page=16, pad=90, max_ctx=3000, max_tokens=800),
    "many-sequences": dict(seqs=[(i % 37, i % 5) for i in range(700)], hq=4, hkv=2, page=16),
    "decoding-64-split": dict(seqs=[(300 + 37 * i, 1) for i in range(64)], hq=16, hkv=2, page=16),
    "even-ragged-decoding": dict(seqs=[(5000, 1), (1, 1), (0, 0), (3000, 1), (127, 1), (700, 1)], hq=32, hkv=8, page=16, pad=2),
    "even-equal-contiguous": dict(seqs=[(4095, 1)] * 8, hq=32, hkv=8),
    "even-chunks-two-m-tiles": dict(seqs=[(4000, 60), (2900, 33), (100, 64), (6000, 1)], hq=16, hkv=4, page=64, layers=2, layer=1),
    "even-40-sequences": dict(seqs=[(0, 1)] * 33 + [(9000, 2), (0, 0), (7000, 1), (256, 1), (6500, 2), (128, 1), (127, 1)],
                              hq=8, hkv=1, page=32),
    "even-uncut": dict(seqs=[(900 + i, 1) for i in range(16)], hq=32, hkv=8, page=128, max_ctx=20000),
    "even-group5": dict(seqs=[(2500, 3), (2600, 50)], hq=10, hkv=2, page=16),
    "cut-decoding-and-chunk": dict(seqs=[(4000, 1), (3, 1), (0, 300), (2500, 1), (6000, 1)], hq=32, hkv=8, page=16, pad=3),
    "cut-chunks-of-blocks": dict(seqs=[(3000, 200), (0, 0), (1500, 333), (40, 1)], hq=16, hkv=4),
    "cut-one-chunk": dict(seqs=[(2500, 130)], hq=16, hkv=2, page=128),
    "cut-short-prompts": dict(seqs=[(0, 512), (0, 100)], hq=8, hkv=8, page=64),
    "cut-34-sequences": dict(seqs=[(0, 1)] * 31 + [(5000, 1), (0, 0), (3000, 150)], hq=8, hkv=1, page=32),
    "cut-200-sequences": dict(seqs=[(37 * i % 3001, 1 - i % 7 // 6) for i in range(200)], hq=4, hkv=1, page=16, pad=4),
    "cut-two-rounds-of-one-length": dict(seqs=[(2600, 1)] * 22, hq=16, hkv=8, page=32),
    "cut-group5-blocks": dict(seqs=[(2000, 120), (2600, 50)], hq=10, hkv=2, page=16),
    "ordered-100": dict(seqs=[(17 * i % 701, 1 + i % 3) for i in range(100)], hq=8, hkv=1, page=32, max_ctx=2000),
    "f32-decoding-split": dict(seqs=[(200 + 11 * i, 1) for i in range(40)], hq=2, hkv=2, d=32, dtype=F32),
    "f32-64": dict(seqs=RAGGED, hq=4, hkv=4, d=64, dtype=F32, pad=2),
    "f32-32-paged": dict(seqs=[(0, 70), (500, 3), (64, 64)], hq=6, hkv=2, d=32, page=16, dtype=F32),
    "f32-128-gqa": dict(seqs=[(33, 65), (0, 200), (900, 1)], hq=8, hkv=2, d=128, page=64, dtype=F32),
    "f32-group80": dict(seqs=[(3, 20)], hq=80, hkv=1, d=64, dtype=F32),
    "f32-long-split": dict(seqs=[(3000, 2)], hq=2, hkv=1, d=64, dtype=F32),
}


@pytest.mark.parametrize("name", list(CASES))
def test_attention_matches_oracle(name):
    kw = dict(CASES[name])
    layer = kw.pop("layer", 0)
    x = Batch(seed=11, **kw)
    x.attend(layer)
    assert int(x.status) == 0
    x.check(layer)


@pytest.mark.parametrize("name", ["gqa-paged16-ragged", "long-split", "f32-64", "f32-long-split"])
def test_attention_without_workspace_and_twice(name):
    """Unsplit calls agree with the oracle too, and a call gives the same bits again (also where another
    call has used its scratch)."""
    x = Batch(seed=12, **CASES[name])
    assert x.attend(workspace=None) == 1
    x.check()
    ws = x.workspace()
    x.out.fill_(7.0)
    launches = x.attend(workspace=ws)
    assert launches == (1 if ws is None else 2)
    x.check()
    first = x.out.clone()
    if ws is not None:
        ws.fill_(255)
    x.attend(workspace=ws)
    assert torch.equal(x.out, first)


def test_attention_scale_and_strided_queries():
    x = Batch([(9, 70), (0, 3)], 8, 2, seed=13)
    wide = torch.full((x.N, 11, 128), float("nan"), dtype=BF16, device=DEV)
    wide[:, :8] = x.q
    x.attend(q=wide[:, :8], scale=0.02)
    x.check(scale=0.02)
    x.out.fill_(7.0)
    x.attend(q=wide[:, :8])
    x.check()


@pytest.mark.parametrize("dtype,d", [(BF16, 128), (F32, 64)])
@pytest.mark.parametrize("value", [float("nan"), float("inf"), float("-inf")])
def test_hidden_values_stay_hidden(dtype, d, value):
    """An infinity or NaN in K and V of a token changes the rows that see it, and no other bit."""
    seqs, at = [(0, 150), (70, 100), (300, 2)], [130, 75, 301]
    x = Batch(seqs, 8, 2, d=d, page=16, dtype=dtype, seed=14)
    x.attend(workspace=None)
    clean = x.out.clone()
    for which in ("v", "k"):
        y = Batch(seqs, 8, 2, d=d, page=16, dtype=dtype, seed=14)
        for b, p in enumerate(at):
            getattr(y, which)[0].view(-1, 2, d)[y.rows[b][p], :, 3:5] = value
        y.attend(workspace=None)
        for b, (c, n) in enumerate(seqs):
            lo, first = y.off[b], y.off[b] + max(0, at[b] - c)
            assert torch.equal(y.out[lo:first], clean[lo:first]), (which, b)
            seen = y.out[first:y.off[b + 1]]
            if which == "v":
                assert not torch.isfinite(seen[:, :, 3:5]).any(), b
                assert torch.isfinite(seen[:, :, 5:]).all() and torch.isfinite(seen[:, :, :3]).all(), b
                if not math.isnan(value):
                    assert (seen[:, :, 3:5] == value).all(), b
            elif math.isnan(value):
                assert torch.isnan(seen).all(), b


@pytest.mark.parametrize("value", [float("nan"), float("inf")])
def test_hidden_values_stay_hidden_in_cut_units(value):
    """The same where the lengths cut a unit: in its last, partly visible key tiles, and in a piece that all rows see."""
    seqs, at = [(4000, 150), (3, 2), (5000, 40)], [4100, 4, 1000]
    x = Batch(seqs, 16, 4, page=16, seed=16)
    assert x.attend() == 2
    clean = x.out.clone()
    for which in ("v", "k"):
        y = Batch(seqs, 16, 4, page=16, seed=16)
        for b, p in enumerate(at):
            getattr(y, which)[0].view(-1, 4, 128)[y.rows[b][p], :, 3:5] = value
        y.attend()
        for b, (c, n) in enumerate(seqs):
            lo, first = y.off[b], y.off[b] + max(0, at[b] - c)
            assert torch.equal(y.out[lo:first], clean[lo:first]), (which, b)
            seen = y.out[first:y.off[b + 1]]
            if which == "v":
                assert torch.isfinite(seen[:, :, 5:]).all() and torch.isfinite(seen[:, :, :3]).all(), b
                assert (torch.isnan(seen[:, :, 3:5]) if math.isnan(value) else seen[:, :, 3:5] == value).all(), b
            elif math.isnan(value):
                assert torch.isnan(seen).all(), b


def test_attention_of_large_scores():
    """Scores of some hundreds, rising and falling along the keys: the running maximum moves in every tile."""
    x = Batch([(0, 300), (600, 40)], 8, 2, seed=15)
    for b in range(2):
        r = x.rows[b]
        ramp = torch.linspace(0.1, 20.0, len(r), device=DEV)
        ramp = ramp if b == 0 else ramp.flip(0)
        x.k[0].view(-1, 2, 128)[r] = (x.k[0].view(-1, 2, 128)[r].float() * ramp[:, None, None]).to(BF16)
    x.attend()
    x.check()


@pytest.mark.parametrize("dtype,d", [(BF16, 128), (F32, 32)])
def test_malformed_sequences_are_reported_and_skipped(dtype, d):
    seqs = [(10, 20), (5, 40), (0, 30), (50, 3)]
    for change in ("ctx", "negative", "tokens", "offset", "capacity"):
        x = Batch(seqs, 4, 2, d=d, page=16, dtype=dtype, seed=16, max_ctx=60, max_tokens=45)
        bad = [1]
        if change == "ctx":
            x.ctx_lens[1] = 61
        elif change == "negative":
            x.ctx_lens[1] = -1
        elif change == "capacity":
            x.ctx_lens[1] = 60   # 60 + 40 positions, the table's row holds 80
            x.prompt = ptd.Prompt(x.token_offsets, x.ctx_lens, x.N, 45, 60)
        elif change == "tokens":
            x.prompt = ptd.Prompt(x.token_offsets, x.ctx_lens, x.N, 39, 60)
        else:
            x.token_offsets[4] = x.N + 1
            bad = [3]
        x.attend()
        assert int(x.status) == ptd.INVALID_BATCH, change
        good = [b for b in range(4) if b not in bad]
        out = x.out.clone()
        for b in bad:
            assert (x.out[x.off[b]:x.off[b + 1]] == 7.0).all(), change
        x.off[-1] = x.N
        x.out = out
        x.check(seqs=good)


@pytest.mark.parametrize("dtype,d", [(BF16, 128), (F32, 32)])
def test_page_outside_the_cache_is_reported(dtype, d):
    x = Batch([(10, 20), (5, 40)], 4, 2, d=d, page=16, dtype=dtype, seed=17)
    for value in (-1, x.num_pages, 2 ** 31 - 1, -2 ** 31):
        x.table[1, 0] = value
        x.status.zero_()
        x.attend()
        assert int(x.status) == ptd.INVALID_BATCH
        x.check(seqs=[0])


# ---------------------------------------------------------------------------------------------------- slots

def _pool(held, table, free, num_pages):
    stack = torch.full((num_pages,), -1, **I32)
    stack[:len(free)] = torch.tensor(free, **I32)
    h = torch.tensor(held, **I32)
    return ptd.PagePool(stack, torch.tensor([len(free)], **I32), h, torch.full_like(h, -9), torch.full((1,), -9, **I32))


def _slots_case(seed, batch, page, longest, num_extra):
    rng = np.random.default_rng(seed)
    ctx = rng.integers(0, longest + 1, batch) * (rng.random(batch) < 0.7)
    new = rng.integers(0, longest + 1, batch) * (rng.random(batch) < 0.8)
    held = -(-ctx // page) + rng.integers(0, 3, batch) * (rng.random(batch) < 0.3)
    need = -(-(ctx + new) // page)
    num = int(max(held.sum(), need.sum())) + num_extra
    width = int(max(held.max(), need.max(), 1)) + 1
    perm = rng.permutation(num).astype(np.int32)
    table, at = np.full((batch, width), -1, np.int32), 0
    for b in range(batch):
        table[b, :held[b]] = perm[at:at + held[b]]
        at += held[b]
    return ctx.tolist(), new.tolist(), held.tolist(), table, perm[at:].tolist(), num


def _small_cache(num_pages, page, table):
    k = torch.zeros((1, num_pages, page, 1, 8), dtype=BF16, device=DEV)
    return ptd.KVCache(k, k.clone(), 1, 8, page, table)


@pytest.mark.parametrize("seed,batch,page,longest,pad", [(1, 1, 16, 40, 0), (2, 7, 16, 100, 3), (3, 513, 32, 20, 0),
                                                         (4, 64, 128, 3000, 11), (5, 8192, 16, 3, 1), (6, 2, 64, 30000, 0)])
def test_slots_with_pages_match_oracle(seed, batch, page, longest, pad):
    ctx, new, held, table, free, num = _slots_case(seed, batch, page, longest, 4)
    off = np.concatenate([[0], np.cumsum(new)])
    N = int(off[-1]) + pad or 1
    t = torch.tensor(table, **I32)
    cache, pool = _small_cache(num, page, t), _pool(held, table, free, num)
    prompt = ptd.Prompt(torch.tensor(off, **I32), torch.tensor(ctx, **I32), N, longest, longest)
    slots, pos, status = torch.full((N,), 5, **I32), torch.full((N,), 5, **I32), torch.zeros(1, **I32)
    want_t, want_held, want_free = oracle.prompt_pages(ctx, new, held, table.tolist(), free, page)
    want_slots, want_pos = oracle.prompt_slots(ctx, new, want_t, page)
    stack = pool.free_pages.clone()
    stack[len(free):len(want_free)] = torch.tensor(want_free[len(free):], **I32)
    for _ in range(2):   # the same state again: the same answer
        assert ptd.prompt_slots(prompt, cache, slots, pos, status, pool) == 1
        torch.cuda.synchronize()
        assert int(status) == 0
        assert t.tolist() == want_t and pool.new_held.tolist() == want_held
        assert int(pool.new_free_count) == len(want_free) and torch.equal(pool.free_pages, stack)
        rest = N - int(off[-1])
        assert slots.tolist() == want_slots + [-1] * rest and pos.tolist() == want_pos + [-1] * rest
    # without the pool, on the finished table
    slots.fill_(5), pos.fill_(5)
    ptd.prompt_slots(prompt, cache, slots, pos, status)
    assert slots.tolist() == want_slots + [-1] * rest and pos.tolist() == want_pos + [-1] * rest and int(status) == 0


def test_slots_of_a_contiguous_cache():
    k = torch.zeros((1, 3, 50, 1, 8), dtype=BF16, device=DEV)
    prompt = ptd.Prompt(torch.tensor([0, 4, 4, 10], **I32), torch.tensor([0, 7, 44], **I32), 12, 6, 44)
    slots, pos, status = torch.zeros(12, **I32), torch.zeros(12, **I32), torch.zeros(1, **I32)
    ptd.prompt_slots(prompt, ptd.KVCache(k, k.clone(), 1, 8), slots, pos, status)
    assert slots.tolist() == [0, 1, 2, 3] + list(range(144, 150)) + [-1, -1] and int(status) == 0
    assert pos.tolist() == [0, 1, 2, 3] + list(range(44, 50)) + [-1, -1]


def test_slots_refused_as_a_whole():
    ctx, new, held, table, free, num = _slots_case(8, 20, 16, 90, 0)
    off = np.concatenate([[0], np.cumsum(new)])
    N = int(off[-1])
    for why in ("pages", "held", "negative", "count", "ctx", "offsets", "twice"):
        t = torch.tensor(table, **I32)
        cache, pool = _small_cache(num, 16, t), _pool(held, table, free, num)
        o, c = torch.tensor(off, **I32), torch.tensor(ctx, **I32)
        max_ctx = 90
        if why == "pages":
            short = sum(-(-(a + b) // 16) - h for a, b, h in zip(ctx, new, held)) - 1
            assert 0 <= short < len(free)
            pool.free_count.fill_(short)
        elif why == "held":
            pool.held[3] = table.shape[1] + 1
        elif why == "negative":
            pool.held[3] = -1
        elif why == "count":
            pool.free_count.fill_(num + 1)
        elif why == "ctx":
            c[5] = 91
        elif why == "offsets":
            o[5] = int(off[4]) - 1 if off[4] > 0 else int(off[-1]) + 1
        else:   # more pages than there are
            c.zero_()
            o.zero_()
            pool.free_count.fill_(num)
        before = (pool.held.clone(), pool.free_count.clone(), pool.free_pages.clone())
        prompt = ptd.Prompt(o, c, N, 90, max_ctx)
        slots, pos, status = torch.full((N,), 5, **I32), torch.full((N,), 5, **I32), torch.zeros(1, **I32)
        ptd.prompt_slots(prompt, cache, slots, pos, status, pool)
        torch.cuda.synchronize()
        assert int(status) == (ptd.NO_PAGES if why == "pages" else ptd.INVALID_BATCH), why
        assert t.tolist() == table.tolist() and torch.equal(pool.free_pages, before[2]), why
        assert torch.equal(pool.new_held, before[0]) and torch.equal(pool.new_free_count, before[1]), why
        assert (slots == -1).all() and (pos == -1).all(), why


def test_slots_without_a_pool_skip_bad_sequences_and_pages():
    t = torch.tensor([[3, 1], [0, 9], [2, -1]], **I32)   # 5 pages
    cache = _small_cache(5, 16, t)
    prompt = ptd.Prompt(torch.tensor([0, 3, 8, 10], **I32), torch.tensor([15, 14, 0], **I32), 10, 5, 20)
    slots, pos, status = torch.zeros(10, **I32), torch.zeros(10, **I32), torch.zeros(1, **I32)
    ptd.prompt_slots(prompt, cache, slots, pos, status)
    assert slots.tolist() == [63, 16, 17, 14, 15, -1, -1, -1, 32, 33] and int(status) == ptd.INVALID_BATCH
    assert pos.tolist() == [15, 16, 17, 14, 15, -1, -1, -1, 0, 1]
    prompt.ctx_lens[0] = 21
    status.zero_()
    t[1, 1] = 4
    ptd.prompt_slots(prompt, cache, slots, pos, status)
    assert slots.tolist() == [-1, -1, -1, 14, 15, 64, 65, 66, 32, 33] and int(status) == ptd.INVALID_BATCH


# ----------------------------------------------------------------------------------------------- rotary append

def _rope_tolerance(x, y, dtype):
    """Rotated pairs: the table's entries are off by 2^-21 (sincosf's 2 ulp, the correction, e^3 / 6 for
    |e| < 2^-7), the products and the sum by 2^-23 of |a| + |b|, then the output's rounding."""
    half = x.shape[-1] // 2
    s = np.abs(x[..., :half]) + np.abs(x[..., half:])
    return np.concatenate([s, s], -1) * (2.0 ** -21 + 2.0 ** -23) + np.abs(y) * (2.0 ** -8 if dtype == BF16 else 2.0 ** -24)


@pytest.mark.parametrize("dtype,hq,hkv,d,page,positions", [
    (BF16, 32, 8, 128, 16, [0, 1, 7, 131071, 4096, 40000]), (F32, 8, 8, 64, 0, [0, 5, 100000, 3]),
    (BF16, 10, 2, 128, 32, list(range(100, 1300))), (BF16, 3, 1, 48, 16, [9, 8, 70000]), (F32, 4, 2, 6, 0, [4, 11, 2]),
    (F32, 32, 8, 128, 64, list(range(50))), (BF16, 4, 4, 256, 16, [33] * 3),
    # more tokens than places for CTAs: rows of several rounds, several tokens a CTA
    (F32, 64, 8, 128, 0, list(range(700))), (BF16, 4, 2, 64, 16, list(range(6500))), (BF16, 2, 1, 32, 0, list(range(12001)))])
@pytest.mark.parametrize("fused", [False, True])
def test_rope_append_matches_oracle(dtype, hq, hkv, d, page, positions, fused):
    n, pad, layers = len(positions), 3, 2
    g = torch.Generator(device=DEV).manual_seed(21)
    rows = 8 * ((n + pad) // 8 + 4)
    shape = (layers, rows * 2 // page + 1, page, hkv, d) if page else (layers, 2, rows, hkv, d)
    kc, vc = (torch.randn(shape, generator=g, device=DEV).to(dtype) for _ in range(2))
    table = torch.zeros((2, 1 << 14), **I32) if page else None
    cache = ptd.KVCache(kc, vc, hkv, d, page, table)
    per_layer = kc[0].numel() // (hkv * d)
    slots = torch.randperm(per_layer, generator=g, device=DEV)[:n + pad].to(torch.int32)
    slots[n:] = -1
    pos = torch.tensor(positions + [-1] * pad, **I32)
    if fused:
        w = torch.randn((n + pad, (hq + 2 * hkv) * d + 8), generator=g, device=DEV).to(dtype)
        q, k, v = (w[:, a * d:b * d].view(n + pad, b - a, d) for a, b in ((0, hq), (hq, hq + hkv), (hq + hkv, hq + 2 * hkv)))
    else:
        q, k, v = (torch.randn((n + pad, h, d), generator=g, device=DEV).to(dtype) for h in (hq, hkv, hkv))
    prompt = ptd.Prompt(torch.tensor([0, n // 2, n], **I32), torch.zeros(2, **I32), n + pad, n, 0)
    status, base = torch.zeros(1, **I32), 500000.0
    k0, v0, qh, kh = kc.clone(), vc.clone(), q.double().cpu().numpy()[:n], k.double().cpu().numpy()[:n]
    q_out = torch.full((n + pad, hq, d), 7.0, dtype=dtype, device=DEV)
    assert ptd.prompt_rope_append(prompt, cache, 1, slots, pos, q, k, v, q_out, base, status) == 1
    torch.cuda.synchronize()
    assert int(status) == 0
    want = oracle.rope(qh, positions, base)
    got = q_out.double().cpu().numpy()
    assert (np.abs(got[:n] - want) <= _rope_tolerance(qh, want, dtype)).all()
    assert (got[n:] == 7.0).all()
    r = slots[:n].long()
    want = oracle.rope(kh, positions, base)
    got = kc[1].view(-1, hkv, d)[r].double().cpu().numpy()
    assert (np.abs(got - want) <= _rope_tolerance(kh, want, dtype)).all()
    assert torch.equal(vc[1].view(-1, hkv, d)[r], v[:n])
    k0[1].view(-1, hkv, d)[r] = kc[1].view(-1, hkv, d)[r]
    v0[1].view(-1, hkv, d)[r] = v[:n]
    assert torch.equal(kc, k0) and torch.equal(vc, v0)       # nothing else was written
    # in place: the same bits
    ptd.prompt_rope_append(prompt, cache, 1, slots, pos, q, k, v, q, base, status)
    assert torch.equal(q[:n], q_out[:n])


def test_rope_append_reports_slots_outside_the_cache():
    kc = torch.zeros((2, 1, 10, 1, 128), dtype=BF16, device=DEV)
    cache = ptd.KVCache(kc, kc.clone(), 1, 128)
    prompt = ptd.Prompt(torch.tensor([0, 4], **I32), torch.zeros(1, **I32), 4, 4, 0)
    x = torch.ones((4, 1, 128), dtype=BF16, device=DEV)
    for bad in (10, -2, 2 ** 31 - 1, -2 ** 31):
        kc.zero_()
        out, status = torch.zeros_like(x), torch.zeros(1, **I32)
        slots = torch.tensor([1, bad, 3, -1], **I32)
        ptd.prompt_rope_append(prompt, cache, 0, slots, torch.arange(4, **I32), x, x, x, out, 1e4, status)
        assert int(status) == ptd.INVALID_BATCH
        assert (kc != 0).view(2, 10, 128).any(-1).tolist() == [[False, True, False, True] + [False] * 6, [False] * 10]
        assert (out != 0).view(4, 128).any(-1).tolist() == [True, False, True, False]


# ------------------------------------------------------------------------------------------------- together

def test_chunks_pages_and_trees_together():
    """Two requests over a paged cache, their prompts admitted in chunks (slots, append, attention per layer), give
    the same outputs as their whole prompts at once on a contiguous cache; a tree that is a chain then sees what one
    more chunk would; a finished request's pages serve the next."""
    g = torch.Generator(device=DEV).manual_seed(31)
    L, hq, hkv, d, page, base = 2, 8, 2, 128, 16, 1e4
    total = [150, 83]
    x = [[torch.randn((n, h, d), generator=g, device=DEV).to(BF16) for h in (hq, hkv, hkv)] for n in total]
    chunks = [[60, 40], [1, 43], [0, 0], [89, 0]]
    num = 16
    shape = (L, num, page, hkv, d)
    kp, vp = (torch.full(shape, float("nan"), dtype=BF16, device=DEV) for _ in range(2))
    table = torch.full((2, 12), -1, **I32)
    cache = ptd.KVCache(kp, vp, hkv, d, page, table)
    free, count = torch.arange(num, **I32), torch.tensor([num], **I32)
    held, status = torch.zeros(2, **I32), torch.zeros(1, **I32)
    done, outs = [0, 0], [[torch.zeros_like(x[b][0]) for b in range(2)] for _ in range(L)]
    for new in chunks:
        N = sum(new) + 2
        off = torch.tensor([0, new[0], sum(new)], **I32)
        prompt = ptd.Prompt(off, torch.tensor(done, **I32), N, 100, 200)
        pool = ptd.PagePool(free, count, held, torch.empty_like(held), torch.empty_like(count))
        slots, pos = torch.empty(N, **I32), torch.empty(N, **I32)
        ptd.prompt_slots(prompt, cache, slots, pos, status, pool)
        held, count = pool.new_held, pool.new_free_count
        q, k, v = (torch.cat([x[b][i][done[b]:done[b] + new[b]] for b in range(2)] + [x[0][i][:2]]) for i in range(3))
        ws = None
        for l in range(L):
            qr, o = torch.empty_like(q), torch.empty_like(q)
            ptd.prompt_rope_append(prompt, cache, l, slots, pos, q, k, v, qr, base, status)
            n = ptd.prompt_attention_workspace_size(prompt, cache, hq)
            ws = torch.empty(max(n, 16), dtype=torch.uint8, device=DEV)
            ptd.prompt_attention(prompt, cache, l, qr, o, status, workspace=ws)
            for b in range(2):
                outs[l][b][done[b]:done[b] + new[b]] = o[int(off[b]):int(off[b + 1])]
        done = [a + b for a, b in zip(done, new)]
    assert done == total and int(status) == 0
    assert held.tolist() == [10, 6] and int(count) == 0
    # whole prompts, contiguous
    kc, vc = (torch.full((L, 2, 160, hkv, d), float("nan"), dtype=BF16, device=DEV) for _ in range(2))
    whole = ptd.KVCache(kc, vc, hkv, d)
    N = sum(total)
    prompt = ptd.Prompt(torch.tensor([0, total[0], N], **I32), torch.zeros(2, **I32), N, max(total), 0)
    slots, pos = torch.empty(N, **I32), torch.empty(N, **I32)
    ptd.prompt_slots(prompt, whole, slots, pos, status)
    q, k, v = (torch.cat([x[b][i] for b in range(2)]) for i in range(3))
    kv = {}
    for l in range(L):
        qr, o = torch.empty_like(q), torch.empty_like(q)
        ptd.prompt_rope_append(prompt, whole, l, slots, pos, q, k, v, qr, base, status)
        ptd.prompt_attention(prompt, whole, l, qr, o, status)
        for b in range(2):
            lo, hi = (0, total[0]) if b == 0 else (total[0], N)
            kb, vb = (c[l, b, :total[b]].double().cpu().numpy() for c in (kc, vc))
            qb = qr[lo:hi].double().cpu().numpy()
            ref, size = oracle.causal_attention(qb, kb, vb, 0)
            tol = _attention_tolerance(qb, kb, vb, ref, size, BF16)
            for got in (o[lo:hi], outs[l][b]):
                assert (np.abs(got.double().cpu().numpy() - ref) <= tol).all()
            kv[l, b] = (kb, vb)
            p = torch.arange(total[b], device=DEV)
            rows = table[b].long()[p // page] * page + p % page
            assert torch.equal(kp[l].view(-1, hkv, d)[rows], kc[l, b, :total[b]])
            assert torch.equal(vp[l].view(-1, hkv, d)[rows], vc[l, b, :total[b]])
    # request 1 is finished; request 0 drafts a chain of 5 nodes over its pages, with the freed ones
    prompt = ptd.Prompt(torch.tensor([0, 5, 5], **I32), torch.tensor([total[0], 0], **I32), 5, 5, 200)
    pool = ptd.PagePool(free, count, held, torch.empty_like(held), torch.empty_like(count))
    slots, pos = torch.empty(5, **I32), torch.empty(5, **I32)
    ptd.prompt_slots(prompt, cache, slots, pos, status, pool)
    assert pool.new_held.tolist() == [10, 0] and int(pool.new_free_count) == 6
    tree = ptd.Tree(torch.tensor([0, 5], **I32), torch.arange(-1, 4, **I32), torch.tensor([total[0]], **I32), 5, 200)
    one = ptd.KVCache(kp, vp, hkv, d, page, table[:1].contiguous())
    q5, k5, v5 = (torch.randn((5, h, d), generator=g, device=DEV).to(BF16) for h in (hq, hkv, hkv))
    qt, qc = q5.clone(), torch.empty_like(q5)
    ptd.prompt_rope_append(prompt, cache, 0, slots, pos, q5, k5, v5, qc, base, status)
    o = torch.empty_like(qc)
    ptd.prompt_attention(prompt, cache, 0, qc, o, status)
    ptd.tree_rope_append(tree, one, 0, qt, hq, k5, v5, base, status)
    assert torch.equal(qt, qc)
    o_tree = torch.empty_like(qt)
    ptd.tree_attention(tree, one, qt, o_tree, hq, status, layer_begin=0, num_layers=1)
    kb, vb = kv[0, 0]
    rows = table[0].long()[torch.arange(150, 155, device=DEV) // page] * page + torch.arange(150, 155, device=DEV) % page
    kb, vb = (np.concatenate([a, c[0].view(-1, hkv, d)[rows].double().cpu().numpy()]) for a, c in ((kb, kp), (vb, vp)))
    ref, size = oracle.causal_attention(qc.double().cpu().numpy(), kb, vb, 150)
    tol = _attention_tolerance(qc.double().cpu().numpy(), kb, vb, ref, size, BF16)
    for got in (o, o_tree):
        assert (np.abs(got.double().cpu().numpy() - ref) <= tol).all()
    assert int(status) == 0


def test_captured_steps_with_changing_lengths():
    """One decoding step captured (slots, append, attention) and replayed while lengths and pages change on the
    device; two graphs that share the scratch, replayed in turn."""
    g = torch.Generator(device=DEV).manual_seed(41)
    hq, hkv, d, page, B, num = 8, 2, 128, 16, 3, 60
    kp, vp = (torch.full((1, num, page, hkv, d), float("nan"), dtype=BF16, device=DEV) for _ in range(2))
    table = torch.full((B, 40), -1, **I32)
    cache = ptd.KVCache(kp, vp, hkv, d, page, table)
    free, count, held = torch.arange(num, **I32), torch.tensor([num], **I32), torch.zeros(B, **I32)
    N, off, ctx = 130, torch.zeros(B + 1, **I32), torch.zeros(B, **I32)
    prompt = ptd.Prompt(off, ctx, N, 128, 600)
    pool = ptd.PagePool(free, count, held, torch.empty_like(held), torch.empty_like(count))
    slots, pos, status = torch.empty(N, **I32), torch.empty(N, **I32), torch.zeros(1, **I32)
    q, qr, o = (torch.zeros((N, hq, d), dtype=BF16, device=DEV) for _ in range(3))
    k, v = (torch.zeros((N, hkv, d), dtype=BF16, device=DEV) for _ in range(2))
    n = ptd.prompt_attention_workspace_size(prompt, cache, hq)
    ws = torch.empty(max(n, 16), dtype=torch.uint8, device=DEV)

    def step(stream):
        ptd.prompt_slots(prompt, cache, slots, pos, status, pool, stream=stream)
        held.copy_(pool.new_held)
        count.copy_(pool.new_free_count)
        ptd.prompt_rope_append(prompt, cache, 0, slots, pos, q, k, v, qr, 1e4, status, stream=stream)
        ptd.prompt_attention(prompt, cache, 0, qr, o, status, workspace=ws, stream=stream)

    graphs = []
    for _ in range(2):
        gr = torch.cuda.CUDAGraph()
        with torch.cuda.graph(gr):
            step(torch.cuda.current_stream())
        graphs.append(gr)
    lens = [0] * B
    for i, new in enumerate([(100, 1, 0), (1, 1, 128), (1, 1, 1), (17, 90, 1), (1, 0, 1)]):
        off.copy_(torch.tensor(np.concatenate([[0], np.cumsum(new)]), dtype=torch.int32))
        ctx.copy_(torch.tensor(lens, dtype=torch.int32))
        for x in (q, k, v):
            x.copy_(torch.randn(x.shape, generator=g, device=DEV).to(BF16))
        o.fill_(7.0)
        graphs[i % 2].replay()
        torch.cuda.synchronize()
        assert int(status) == 0
        at = 0
        for b in range(B):
            lens[b] += new[b]
            if new[b]:
                p = torch.arange(lens[b], device=DEV)
                rows = table[b].long()[p // page] * page + p % page
                kb, vb = (c[0].view(-1, hkv, d)[rows].double().cpu().numpy() for c in (kp, vp))
                qb = qr[at:at + new[b]].double().cpu().numpy()
                ref, size = oracle.causal_attention(qb, kb, vb, lens[b] - new[b])
                tol = _attention_tolerance(qb, kb, vb, ref, size, BF16)
                assert (np.abs(o[at:at + new[b]].double().cpu().numpy() - ref) <= tol).all()
            at += new[b]
        assert (o[at:] == 7.0).all()


def test_captured_decoding_is_cut_anew_at_each_replay():
    """One captured decoding call over lengths that change on the device: cut into shares or not, sequences that drop
    out, and one out of range, whose row stays as it was."""
    x = Batch([(6000, 1)] * 5, 16, 4, page=32, pad=3, seed=70)
    ws = x.workspace()
    gr = torch.cuda.CUDAGraph()
    with torch.cuda.graph(gr):
        assert ptd.prompt_attention(x.prompt, x.cache, 0, x.q, x.out, x.status, workspace=ws) == 2
    for ctx, new in (([6000] * 5, [1] * 5), ([0, 5999, 127, 2000, 128], [1] * 5), ([3, 1, 0, 100, 20], [1] * 5),
                     ([4000, 0, 0, 10, 900], [1, 0, 0, 1, 1]), ([0] * 5, [0] * 5), ([700, 6001, 5000, 3000, 9], [1] * 5)):
        bad = [c > 6000 for c in ctx]
        off = np.concatenate([[0], np.cumsum(new)])
        x.ctx_lens.copy_(torch.tensor(ctx, dtype=torch.int32))
        x.token_offsets.copy_(torch.tensor(off, dtype=torch.int32))
        x.out.fill_(7.0)
        x.status.zero_()
        ws.fill_(255)
        gr.replay()
        torch.cuda.synchronize()
        assert int(x.status) == (ptd.INVALID_BATCH if any(bad) else 0)
        for b in range(5):
            if new[b] and bad[b]:
                assert (x.out[off[b]] == 7.0).all()
            elif new[b]:
                k, v = x.kv(b)
                q = x.q[off[b]:off[b] + 1].double().cpu().numpy()
                ref, size = oracle.causal_attention(q, k, v, ctx[b])
                tol = _attention_tolerance(q, k, v, ref, size, BF16)
                assert (np.abs(x.out[off[b]:off[b] + 1].double().cpu().numpy() - ref) <= tol).all()
        assert (x.out[off[-1]:] == 7.0).all()


@pytest.mark.parametrize("dtype,hkv,d,capacity", [(BF16, 8, 128, 2_200_000), (F32, 8, 64, 4_300_000)])
def test_offsets_past_32_bits(dtype, hkv, d, capacity):
    """The second sequence of a contiguous cache begins 2^31 elements on: slots, append and attention."""
    hq, ctx, new = 2 * hkv, [5, 130], [1, 3]
    kc, vc = (torch.empty((1, 2, capacity, hkv, d), dtype=dtype, device=DEV) for _ in range(2))
    assert kc[0, 0].numel() > 2 ** 31
    g = torch.Generator(device=DEV).manual_seed(80)
    rand = lambda *s: torch.randn(s, generator=g, device=DEV).to(dtype)
    for b in range(2):
        for c in (kc, vc):
            c[0, b, :ctx[b]] = rand(ctx[b], hkv, d)
    cache = ptd.KVCache(kc, vc, hkv, d)
    prompt = ptd.Prompt(torch.tensor([0, 1, 4], **I32), torch.tensor(ctx, **I32), 4, 3, 130)
    slots, pos, status = torch.empty(4, **I32), torch.empty(4, **I32), torch.zeros(1, **I32)
    q, k, v = rand(4, hq, d), rand(4, hkv, d), rand(4, hkv, d)
    out = torch.empty_like(q)
    ptd.prompt_slots(prompt, cache, slots, pos, status)
    ptd.prompt_rope_append(prompt, cache, 0, slots, pos, q, k, v, q, 1e4, status)
    n = ptd.prompt_attention_workspace_size(prompt, cache, hq)
    ptd.prompt_attention(prompt, cache, 0, q, out, status, workspace=torch.empty(max(n, 16), dtype=torch.uint8, device=DEV))
    torch.cuda.synchronize()
    assert int(status) == 0
    assert slots.tolist() == [5, capacity + 130, capacity + 131, capacity + 132] and pos.tolist() == [5, 130, 131, 132]
    for b, rows in ((0, slice(0, 1)), (1, slice(1, 4))):
        assert torch.equal(vc[0, b, ctx[b]:ctx[b] + new[b]], v[rows])
        kb, vb, qb = (x.double().cpu().numpy() for x in (kc[0, b, :ctx[b] + new[b]], vc[0, b, :ctx[b] + new[b]], q[rows]))
        want = oracle.rope(k[rows].double().cpu().numpy(), pos[rows].tolist(), 1e4)
        assert (np.abs(kb[ctx[b]:] - want) <= _rope_tolerance(k[rows].double().cpu().numpy(), want, dtype)).all()
        ref, size = oracle.causal_attention(qb, kb, vb, ctx[b])
        tol = _attention_tolerance(qb, kb, vb, ref, size, dtype)
        assert (np.abs(out[rows].double().cpu().numpy() - ref) <= tol).all()


def test_calls_on_two_streams():
    """Batches with scratch of their own on two streams at once."""
    xs = [Batch([(3000 + 500 * i, 2), (40, 9)], 8, 2, page=16, seed=50 + i) for i in range(2)]
    streams = [torch.cuda.Stream() for _ in xs]
    ws = [x.workspace() for x in xs]
    torch.cuda.synchronize()
    for _ in range(5):
        for x, s, w in zip(xs, streams, ws):
            ptd.prompt_attention(x.prompt, x.cache, 0, x.q, x.out, x.status, workspace=w, stream=s)
    torch.cuda.synchronize()
    for x in xs:
        assert int(x.status) == 0
        x.check()


def test_binding_refuses_wrong_tensors():
    x = Batch([(3, 4)], 8, 2, seed=60)
    call = lambda q=x.q, out=x.out, status=x.status: ptd.prompt_attention(x.prompt, x.cache, 0, q, out, status)
    with pytest.raises(TypeError):
        call(q=x.q.float())
    with pytest.raises(ValueError):
        call(q=x.q[:3])
    with pytest.raises(ValueError):
        call(q=x.q.transpose(0, 1).contiguous().transpose(0, 1))
    with pytest.raises(ValueError):
        call(q=x.q.cpu())
    with pytest.raises(ValueError):
        call(out=x.out[:, ::2])
    with pytest.raises(TypeError):
        call(out=x.out.float())
    with pytest.raises(TypeError):
        call(status=x.status.float())
    with pytest.raises(ValueError):
        ptd.prompt_slots(x.prompt, x.cache, torch.zeros(3, **I32), torch.zeros(4, **I32), x.status)
    assert int(x.status) == 0 and (x.out == 7.0).all()


def test_native_and_ctypes_paths_agree(monkeypatch):
    """Each prompt call is taken natively (kernels launched, not None), and gives what the ctypes path gives."""
    calls, taken = ptd._native(), {}

    class Record:
        def __getattr__(self, name):
            def call(*a):
                taken[name] = getattr(calls, name)(*a)
                return taken[name]

            return call

    class Refuse:
        def __getattr__(self, name):
            return lambda *a: None

    def run_all():
        x = Batch([(30, 40), (0, 3), (700, 1)], 8, 2, page=16, seed=70, pad=2)
        free = torch.arange(x.num_pages, **I32)
        held = torch.tensor([2, 0, 44], **I32)
        pool = ptd.PagePool(free, torch.tensor([3], **I32), held, torch.empty_like(held), torch.zeros(1, **I32))
        slots, pos = torch.empty(x.N, **I32), torch.empty(x.N, **I32)
        n = [ptd.prompt_slots(x.prompt, x.cache, slots, pos, x.status, pool), ptd.prompt_slots(x.prompt, x.cache, slots, pos, x.status)]
        q, k, v = x.q, x.q[:, :2].contiguous(), x.q[:, 2:4].contiguous()
        out = torch.zeros_like(q)
        n.append(ptd.prompt_rope_append(x.prompt, x.cache, 0, slots, pos, q, k, v, out, 1e4, x.status))
        x.q = out
        n.append(x.attend())
        assert int(x.status) == ptd.NO_PAGES   # three pages are too few: refused, then slots of the table as it is
        return n, [slots, pos, pool.new_held, x.k.nan_to_num(), x.v.nan_to_num(), out, x.out.nan_to_num()]

    monkeypatch.setattr(ptd, "_calls", Record())
    native = run_all()
    assert set(taken) == {"prompt_slots", "prompt_rope_append", "prompt_attention"} and all(r > 0 for r in taken.values())
    monkeypatch.setattr(ptd, "_calls", Refuse())
    plain = run_all()
    assert native[0] == plain[0]
    for i, (a, b) in enumerate(zip(native[1], plain[1])):
        assert torch.equal(a, b), i


@pytest.mark.parametrize("seqs", [
    # cut by the lengths: some shares begin at a key tile that only the second M tile sees, a unit with both follows
    [(128 * (13 + 5 * i % 7) - 40, 64) for i in range(20)],
    # whole units, several a CTA, the second M tile one key tile longer
    [(88, 64)] * 90], ids=["cut", "whole"])
def test_units_whose_second_m_tile_sees_more(seqs):
    x = Batch(seqs, 16, 4, page=32, seed=71)
    for _ in range(3):
        x.out.fill_(7.0)
        x.attend()
        assert int(x.status) == 0
        x.check()


PI = decimal.Decimal("3.14159265358979323846264338327950288419716939937510582097494459")


def _exact_rope(x, positions, base):
    """The rotation with angles of 60 digits.  An entry of the kernel's table is off by sincospif's 1 ulp (2^-24), the
    rounding of its correction (2^-25) and 2^-32 turns, so below 2^-23, and by p times a frequency's error
    (2^-53 of the power, and a little more where 2j/D is rounded): p 2^-52.  The products and their sum add 2^-23."""
    with decimal.localcontext(decimal.Context(prec=60)):
        half = x.shape[-1] // 2
        freq = [decimal.Decimal(base) ** (decimal.Decimal(-2 * j) / (2 * half)) for j in range(half)]
        angle = np.array([[float(p * f % (2 * PI)) for f in freq] for p in positions])
    c, s = np.cos(angle)[:, None, :], np.sin(angle)[:, None, :]
    a, b = x[..., :half], x[..., half:]
    table = (2.0 ** -23 + np.array(positions, float) * 2.0 ** -52)[:, None, None]
    size = (np.abs(a) + np.abs(b)) * (table + 2.0 ** -23)
    return np.concatenate([a * c - b * s, a * s + b * c], -1), np.concatenate([size, size], -1)


FAR = [0, 1, 2 ** 17, 2 ** 18 + 1, 2 ** 19, 2 ** 20, 2 ** 20 + 3, 2 ** 22 + 5, 2 ** 23 + 1, 2 ** 24 + 1, 2 ** 27 + 33, 2 ** 30 - 1]


@pytest.mark.parametrize("base", [10000.0, 500000.0])
@pytest.mark.parametrize("dtype,hq,hkv,d", [(BF16, 2, 1, 128), (F32, 2, 1, 128), (F32, 2, 2, 64), (F32, 2, 2, 6), (BF16, 1, 1, 256)])
def test_far_positions_are_rotated_exactly(dtype, hq, hkv, d, base):
    n = len(FAR)
    g = torch.Generator(device=DEV).manual_seed(22)
    kc, vc = (torch.zeros((1, 1, n, hkv, d), dtype=dtype, device=DEV) for _ in range(2))
    q, k, v = (torch.randn((n, h, d), generator=g, device=DEV).to(dtype) for h in (hq, hkv, hkv))
    prompt = ptd.Prompt(torch.tensor([0, n], **I32), torch.zeros(1, **I32), n, n, 0)
    slots, pos, status, out = torch.arange(n, **I32), torch.tensor(FAR, **I32), torch.zeros(1, **I32), torch.empty_like(q)
    ptd.prompt_rope_append(prompt, ptd.KVCache(kc, vc, hkv, d), 0, slots, pos, q, k, v, out, base, status)
    assert int(status) == 0
    for x, got in ((q, out), (k, kc[0, 0])):
        want, tol = _exact_rope(x.double().cpu().numpy(), FAR, base)
        tol += np.abs(want) * (2.0 ** -8 if dtype == BF16 else 2.0 ** -24)
        assert (np.abs(got.double().cpu().numpy() - want) <= tol).all()


def test_far_trees_are_rotated_exactly():
    """A tree behind 2^24 + 1 committed tokens: the same table as a prompt's."""
    ctx, hq, hkv, d, base = 2 ** 24 + 1, 2, 1, 8, 10000.0
    kc, vc = (torch.zeros((1, 1, ctx + 8, hkv, d), device=DEV) for _ in range(2))
    g = torch.Generator(device=DEV).manual_seed(23)
    q, k, v = (torch.randn((4, h, d), generator=g, device=DEV) for h in (hq, hkv, hkv))
    status, before = torch.zeros(1, **I32), q.double().cpu().numpy()
    tree = ptd.Tree(torch.tensor([0, 4], **I32), torch.tensor([-1, 0, 0, 1], **I32), torch.tensor([ctx], **I32), 4, ctx)
    ptd.tree_rope_append(tree, ptd.KVCache(kc, vc, hkv, d), 0, q, hq, k, v, base, status)
    assert int(status) == 0
    pos = [ctx, ctx + 1, ctx + 1, ctx + 2]
    for x, got in ((before, q), (k.double().cpu().numpy(), kc[0, 0, ctx:ctx + 4])):
        want, tol = _exact_rope(x, pos, base)
        assert (np.abs(got.double().cpu().numpy() - want) <= tol + np.abs(want) * 2.0 ** -24).all()


def test_slots_of_small_and_large_batches_from_two_threads():
    """Batches that need 54 KB and 160 KB of shared memory, from two threads at once: every call is enqueued."""
    failed, sizes = [], (2700, 8192)

    def work(batch):
        try:
            stream = torch.cuda.Stream()
            with torch.cuda.stream(stream):
                table = torch.arange(batch, **I32).view(batch, 1)
                cache = _small_cache(batch, 16, table)
                held = torch.ones(batch, **I32)
                pool = ptd.PagePool(torch.full((batch,), -1, **I32), torch.zeros(1, **I32), held, torch.empty_like(held),
                                    torch.zeros(1, **I32))
                prompt = ptd.Prompt(torch.arange(batch + 1, **I32), torch.full((batch,), 3, **I32), batch, 1, 3)
                slots, pos, status = torch.empty(batch, **I32), torch.empty(batch, **I32), torch.zeros(1, **I32)
                for _ in range(3000):
                    ptd.prompt_slots(prompt, cache, slots, pos, status, pool)
                stream.synchronize()
                assert int(status) == 0 and torch.equal(slots, torch.arange(batch, **I32) * 16 + 3)
        except Exception as e:
            failed.append((batch, repr(e)))

    threads = [threading.Thread(target=work, args=(b,)) for b in sizes for _ in range(2)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not failed


def test_batches_that_are_not_the_caches_are_refused():
    """Two prompts into a contiguous cache of three sequences, or of one; a block table with too few rows."""
    x, y = Batch([(3, 4), (0, 2)], 8, 2, seed=61), Batch([(3, 4), (0, 2)], 8, 2, page=16, seed=61)
    slots, pos = torch.full((x.N,), 5, **I32), torch.full((x.N,), 5, **I32)
    caches = [ptd.KVCache(x.k.repeat(2, 2, 1, 1, 1)[:, :n].contiguous(),
                          x.v.repeat(2, 2, 1, 1, 1)[:, :n].contiguous(), 2, 128) for n in (1, 3)]
    caches.append(ptd.KVCache(y.k, y.v, 2, 128, 16, y.table[:1].contiguous()))
    k = x.q[:, :2].contiguous()
    for cache in caches:
        for call in (lambda: ptd.prompt_slots(x.prompt, cache, slots, pos, x.status),
                     lambda: ptd.prompt_rope_append(x.prompt, cache, 0, slots, pos, x.q, k, k, x.out, 1e4, x.status),
                     lambda: ptd.prompt_attention(x.prompt, cache, 0, x.q, x.out, x.status)):
            with pytest.raises(ValueError, match="sequences"):
                call()
    torch.cuda.synchronize()
    assert int(x.status) == 0 and (x.out == 7.0).all() and (slots == 5).all() and (pos == 5).all()
    # more rows in the table than sequences in the batch are fine
    more = ptd.KVCache(y.k, y.v, 2, 128, 16, torch.cat([y.table, torch.full_like(y.table[:1], -1)]))
    y.cache = more
    y.attend()
    y.check()


def test_rotated_queries_beside_their_inputs_and_overlaps():
    """q_out may lie between the rows of q, k and v of one wide buffer, or be q; on part of them it is refused, as is an
    attention whose output or scratch lies on what it reads."""
    n, hq, hkv, d = 40, 8, 2, 128
    g = torch.Generator(device=DEV).manual_seed(62)
    w = torch.randn((n, (2 * hq + 2 * hkv) * d), generator=g, device=DEV).to(BF16)
    q, k, v, out = (w[:, a * d:b * d].view(n, b - a, d) for a, b in ((0, 8), (8, 10), (10, 12), (12, 20)))
    kc, vc = (torch.zeros((1, 1, n + 3000, hkv, d), dtype=BF16, device=DEV) for _ in range(2))
    cache = ptd.KVCache(kc, vc, hkv, d)
    prompt = ptd.Prompt(torch.tensor([0, n], **I32), torch.zeros(1, **I32), n, n, 0)
    slots, pos, status = torch.arange(n, **I32), torch.arange(n, **I32), torch.zeros(1, **I32)
    before, want = w.clone(), torch.empty((n, hq, d), dtype=BF16, device=DEV)
    ptd.prompt_rope_append(prompt, cache, 0, slots, pos, q, k, v, want, 1e4, status)
    ptd.prompt_rope_append(prompt, cache, 0, slots, pos, q, k, v, out, 1e4, status)
    assert torch.equal(out, want) and torch.equal(w[:, :12 * d], before[:, :12 * d])
    for on in (w[:, 4 * d:12 * d], w[:, 6 * d:14 * d], w[:, 11 * d:19 * d]):
        with pytest.raises(ptd.PtdError):
            ptd.prompt_rope_append(prompt, cache, 0, slots, pos, q, k, v, on.view(n, hq, d), 1e4, status)
    flat = w.view(-1)
    with pytest.raises(ptd.PtdError):
        ptd.prompt_attention(prompt, cache, 0, q, flat[4 * d:4 * d + n * hq * d].view(n, hq, d), status)
    with pytest.raises(ptd.PtdError):
        ptd.prompt_attention(prompt, cache, 0, q, kc.view(-1)[d:d + n * hq * d].view(n, hq, d), status)
    torch.cuda.synchronize()
    assert torch.equal(w[:, :12 * d], before[:, :12 * d]) and int(status) == 0
    far = ptd.Prompt(torch.tensor([0, 1], **I32), torch.tensor([2900], **I32), 1, 1, 2900)
    size = ptd.prompt_attention_workspace_size(far, cache, hq)
    assert size > 0
    room = torch.zeros(hq * d + size // 2, dtype=BF16, device=DEV)   # a row of queries, then the scratch
    one, query = torch.zeros((1, hq, d), dtype=BF16, device=DEV), room[:hq * d].view(1, hq, d)
    with pytest.raises(ptd.PtdError):
        ptd.prompt_attention(far, cache, 0, query, one, status, workspace=room[:size // 2])
    ptd.prompt_attention(far, cache, 0, query, one, status, workspace=room[hq * d:])
    torch.cuda.synchronize()
    assert int(status) == 0


def test_a_unit_of_some_seconds():
    """One token behind 2^29 positions without scratch: a single CTA reads them all (two pages, one after the other over and
    over), some seconds long, while its roles without work wait.  The scores of the first page are 128, all others 0,
    so that the others' weights are 0 in fp32 (e^-128) and the output is the mean of the first page's 128 values."""
    ctx, page = 2 ** 29, 128
    table = torch.full((1, ctx // page + 1), 1, **I32)
    table[0, 0] = 0
    g = torch.Generator(device=DEV).manual_seed(63)
    k, v = torch.zeros((1, 2, page, 1, 128), dtype=BF16, device=DEV), torch.randn((1, 2, page, 1, 128), generator=g, device=DEV).to(BF16)
    k[0, 0] = 1.0
    q, out, status = torch.ones((1, 1, 128), dtype=BF16, device=DEV), torch.zeros((1, 1, 128), dtype=BF16, device=DEV), torch.zeros(1, **I32)
    prompt = ptd.Prompt(torch.tensor([0, 1], **I32), torch.tensor([ctx], **I32), 1, 1, ctx)
    a, b = (torch.cuda.Event(enable_timing=True) for _ in range(2))
    a.record()
    assert ptd.prompt_attention(prompt, ptd.KVCache(k, v, 1, 128, page, table), 0, q, out, status, scale=1.0) == 1
    b.record()
    torch.cuda.synchronize()
    assert int(status) == 0
    want = v[0, 0, :, 0].double().mean(0)
    # 128 products summed in fp32 by truncation, and the output's rounding
    tol = 128 * 2.0 ** -23 * v[0, 0, :, 0].double().abs().mean(0) + 2.0 ** -8 * want.abs() + 1e-30
    assert ((out[0, 0].double() - want).abs() <= tol).all()
    assert a.elapsed_time(b) > 2000.0   # longer than the waits between steps last
