"""The operators around several continuations without a GPU: the host's refusals, what the native calls take, and the
binding's own checks."""
import ctypes
import math
import os

import numpy as np
import pytest

import oracle

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
A = 1 << 30
COUNTS = {"prompt_norm_rope_append": 15, "tree_norm_rope_append": 14, "token_logprobs": 9, "lm_head_logprobs": 11, "page_fork": 8}


@pytest.fixture(scope="module")
def lib():
    import __graft_entry__

    __graft_entry__.build()
    from paper_2607_10661_gb300 import ptd

    return ptd.lib()


def _cache(ptd, page=16, dtype=None, hkv=8, d=128, layers=2, num_pages=40, max_pages=10, k=2 * A, v=3 * A):
    return ptd._Cache(k, v, ptd.BF16 if dtype is None else dtype, layers, hkv, d, page, 0 if page else 300, num_pages if page else 0,
                      A + 8192 if page else None, max_pages if page else 0)


def test_prompt_norm_rope_append_refusals(lib):
    from paper_2607_10661_gb300 import ptd

    row, kv = 32 * 128 * 2, 1024 * 2

    def call(cache=None, layer=0, slots=4 * A, positions=5 * A, q=7 * A, qs=4096, hq=32, k=8 * A, ks=1024, v=9 * A, vs=1024,
             wq=11 * A, wk=12 * A, eps=1e-6, base=1e4, out=10 * A, outs=4096, status=6 * A, prompt=None):
        prompt = prompt or ptd._Prompt(2, 10, 8, 100, A, A + 4096)
        return lib.ptd_prompt_norm_rope_append(ctypes.byref(prompt), ctypes.byref(cache or _cache(ptd)), layer, slots, positions, q,
                                               qs, hq, k, ks, v, vs, wq, wk, eps, base, out, outs, status, None)

    for kw in (dict(layer=-1), dict(layer=2), dict(slots=None), dict(positions=None), dict(q=None), dict(k=None),
               dict(v=None), dict(out=None), dict(status=None), dict(wq=None), dict(wk=None), dict(eps=-1e-9), dict(eps=float("nan")),
               dict(eps=float("inf")), dict(wq=11 * A + 1), dict(wk=12 * A + 1), dict(qs=4095), dict(ks=1023), dict(vs=0),
               dict(outs=-4096), dict(hq=30), dict(hq=0), dict(base=1.0), dict(base=float("nan")), dict(q=7 * A + 1),
               dict(cache=_cache(ptd, d=264), qs=10**6, outs=10**6, ks=10**6, vs=10**6),
               dict(prompt=ptd._Prompt(0, 10, 8, 100, A, A + 4096))):
        assert call(**kw) == ptd.INVALID_ARG, kw
    # what is written meets what is read: q_out, the status, the cache
    layers = 2 * 40 * 16 * kv
    for kw in (dict(out=7 * A + row), dict(out=8 * A), dict(out=9 * A + kv), dict(out=11 * A), dict(out=12 * A - row), dict(out=4 * A),
               dict(out=5 * A + 16), dict(status=11 * A + 4), dict(status=12 * A), dict(status=4 * A + 8), dict(out=2 * A),
               dict(q=2 * A + layers - row), dict(k=3 * A), dict(v=2 * A + 64), dict(wq=3 * A + layers - 64), dict(slots=2 * A),
               dict(positions=3 * A + 8), dict(cache=_cache(ptd, v=2 * A + 64))):
        assert call(**kw) == ptd.INVALID_ARG, kw
    assert call(hq=2**24 - 16, qs=2**31, outs=2**31) == ptd.UNSUPPORTED
    assert call(prompt=ptd._Prompt(8193, 10, 8, 100, A, A + 4096)) == ptd.UNSUPPORTED


def test_prompt_norm_rope_append_refuses_a_status_on_other_memory(lib):
    """dev_status is written: it lies on no input, not on q_out and not in the cache."""
    from paper_2607_10661_gb300 import ptd

    row, cache_bytes = 32 * 128 * 2, 2 * 40 * 16 * 1024 * 2

    def call(status, out=10 * A):
        prompt = ptd._Prompt(2, 10, 8, 100, A, A + 4096)
        return lib.ptd_prompt_norm_rope_append(ctypes.byref(prompt), ctypes.byref(_cache(ptd)), 0, 4 * A, 5 * A, 7 * A, 4096, 32, 8 * A,
                                               1024, 9 * A, 1024, 11 * A, 12 * A, 1e-6, 1e4, out, 4096, status, None)

    for status in (2 * A, 2 * A + cache_bytes - 4, 3 * A + 64, 7 * A, 7 * A + 10 * row - 4, 8 * A, 9 * A + 16, 10 * A, 11 * A, 12 * A + 252,
                   4 * A + 36, 5 * A):
        assert call(status) == ptd.INVALID_ARG, hex(status)
    assert call(7 * A + 8, out=7 * A) == ptd.INVALID_ARG   # in place too


def test_tree_norm_rope_append_refusals(lib):
    from paper_2607_10661_gb300 import ptd

    n, q, kv = 20, 2 * 20 * 32 * 128 * 2, 2 * 20 * 8 * 128 * 2

    def call(cache=None, layer=0, layers=2, hq=32, qp=7 * A, k=8 * A, v=9 * A, wq=11 * A, wk=12 * A, eps=1e-6, base=1e4, out=10 * A,
             pos=5 * A, status=6 * A, tree=None):
        tree = tree or ptd._Tree(2, n, 16, 100, A, A + 4096, A + 12288)
        return lib.ptd_tree_norm_rope_append(ctypes.byref(tree), ctypes.byref(cache or _cache(ptd)), layer, layers, qp, hq, k, v, wq,
                                             wk, eps, base, out, pos, status, None)

    for kw in (dict(layer=-1), dict(layer=1), dict(layers=0), dict(layers=3), dict(qp=None), dict(k=None), dict(v=None), dict(out=None),
               dict(status=None), dict(wq=None), dict(wk=None), dict(eps=-1.0), dict(eps=float("nan")), dict(hq=30), dict(hq=0),
               dict(base=1.0), dict(qp=7 * A + 1), dict(out=10 * A + 1), dict(wq=11 * A + 1), dict(tree=ptd._Tree(0, n, 16, 100, A, A, A)),
               # overlaps
               dict(out=7 * A + 16), dict(out=7 * A + q - 16), dict(out=8 * A), dict(out=9 * A + kv - 16), dict(out=11 * A),
               dict(out=12 * A), dict(out=2 * A), dict(out=3 * A + 64), dict(pos=7 * A), dict(pos=10 * A + 64), dict(pos=A + 4096),
               dict(status=5 * A + 76), dict(status=A), dict(k=2 * A), dict(v=3 * A), dict(wk=2 * A + 32), dict(out=A + 4096 - q + 4)):
        assert call(**kw) == ptd.INVALID_ARG, kw
    assert call(hq=2**24 - 16) == ptd.UNSUPPORTED
    assert call(cache=_cache(ptd, page=24)) == ptd.UNSUPPORTED


def test_token_logprobs_refusals(lib):
    from paper_2607_10661_gb300 import ptd

    def call(logits=2 * A, dtype=None, rows=5, vocab=1000, stride=1000, tokens=3 * A, T=1.0, k=4, lp=4 * A, en=5 * A, idx=6 * A,
             val=7 * A, status=8 * A):
        return lib.ptd_token_logprobs(logits, ptd.BF16 if dtype is None else dtype, rows, vocab, stride, tokens, T, k, lp, en, idx,
                                      val, status, None)

    for kw in (dict(logits=None), dict(dtype=2), dict(dtype=-1), dict(rows=0), dict(rows=-1), dict(vocab=0), dict(vocab=3), dict(stride=999),
               dict(tokens=None), dict(T=0.0), dict(T=-1.0), dict(T=float("nan")), dict(T=float("inf")), dict(T=1e-39), dict(k=-1),
               dict(k=17), dict(lp=None), dict(idx=None), dict(val=None), dict(status=None), dict(logits=2 * A + 1),
               dict(logits=2 * A + 2, dtype=0), dict(stride=2**61), dict(rows=2**40, stride=2**30),
               # overlaps
               dict(lp=2 * A + 4000), dict(en=4 * A + 16), dict(idx=3 * A), dict(val=6 * A + 76), dict(status=7 * A + 76),
               dict(status=2 * A + 9996), dict(lp=3 * A + 16), dict(en=5 * A, val=5 * A)):
        assert call(**kw) == ptd.INVALID_ARG, kw
    assert call(rows=2**30 + 1) == ptd.UNSUPPORTED and call(vocab=2**30 + 1, stride=2**31) == ptd.UNSUPPORTED


def test_lm_head_logprobs_refusals(lib):
    from paper_2607_10661_gb300 import ptd

    size = lib.ptd_lm_head_logprobs_workspace_size
    need = size(300, 1000, 4)
    assert need > 0 and size(0, 1000, 4) == size(300, 0, 4) == size(300, 1000, -1) == size(300, 1000, 17) == 0
    assert size(2**22 + 1, 1000, 4) == size(300, 2**30 + 1, 4) == 0 and size(300, 1000, 0) < need < size(300, 1000, 16)

    def call(h=2 * A, rows=300, hs=512, w=3 * A, vocab=1000, ws=512, d=512, tokens=4 * A, T=1.0, k=4, lp=5 * A, en=6 * A, idx=7 * A,
             val=8 * A, scratch=9 * A, nbytes=need, status=10 * A):
        return lib.ptd_lm_head_logprobs(h, rows, hs, w, vocab, ws, d, tokens, T, k, lp, en, idx, val, scratch, nbytes, status, None)

    for kw in (dict(h=None), dict(w=None), dict(rows=0), dict(d=0), dict(d=96), dict(d=576), dict(hs=511), dict(ws=511), dict(hs=516),
               dict(ws=516), dict(vocab=3), dict(vocab=0), dict(h=2 * A + 8), dict(w=3 * A + 8), dict(tokens=None), dict(T=0.0),
               dict(T=float("nan")), dict(k=-1), dict(k=17), dict(lp=None), dict(idx=None), dict(val=None), dict(status=None),
               dict(hs=2**60), dict(ws=2**60),
               # overlaps
               dict(lp=2 * A + 64), dict(en=3 * A), dict(idx=4 * A + 16), dict(val=7 * A + 16), dict(status=9 * A + 64),
               dict(lp=9 * A + need - 4), dict(scratch=2 * A), dict(scratch=3 * A + 1024), dict(scratch=4 * A - need + 16)):
        assert call(**kw) == ptd.INVALID_ARG, kw
    for kw in (dict(scratch=None), dict(nbytes=need - 1), dict(scratch=9 * A + 8)):
        assert call(**kw) == ptd.WORKSPACE, kw
    assert call(rows=2**22 + 1) == ptd.UNSUPPORTED and call(vocab=2**30 + 1) == ptd.UNSUPPORTED


def test_lm_head_logprobs_refuses_rows_whose_tile_outlasts_a_wait(lib):
    """A tile's product is waited for at most 2 s: 4 MMAs of 0.34 us per 64 columns, 0.36 s at the limit."""
    from paper_2607_10661_gb300 import ptd

    need = lib.ptd_lm_head_logprobs_workspace_size(1, 5, 0)
    for d in (2**26 + 64, 2**28, 2**31 - 64):
        assert lib.ptd_lm_head_logprobs(16 * A, 1, d, 32 * A, 5, d, d, 3 * A, 1.0, 0, 4 * A, None, None, None, 5 * A, need, 6 * A,
                                        None) == ptd.UNSUPPORTED


def test_page_fork_refusals(lib):
    from paper_2607_10661_gb300 import ptd

    def sets(batch=3, table=4 * A, held=5 * A, free=6 * A, count=7 * A, to_batch=5, new_table=8 * A, new_held=9 * A, new_free=10 * A,
             new_count=11 * A):
        return ptd._PageSet(batch, table, held, free, count), ptd._PageSet(to_batch, new_table, new_held, new_free, new_count)

    def size(cache, s):
        return lib.ptd_page_fork_workspace_size(ctypes.byref(cache), ctypes.byref(s[0]), ctypes.byref(s[1]))

    need = size(_cache(ptd), sets())
    assert need > 0 and size(_cache(ptd, page=0), sets()) == 0 and size(_cache(ptd), sets(batch=0)) == 0

    def call(cache=None, parents=12 * A, lens=13 * A, ws=14 * A, nbytes=need, status=15 * A, **kw):
        s = sets(**kw)
        return lib.ptd_page_fork(ctypes.byref(cache or _cache(ptd)), ctypes.byref(s[0]), ctypes.byref(s[1]), parents, lens, ws, nbytes,
                                 status, None)

    for kw in (dict(cache=_cache(ptd, page=0)), dict(batch=0), dict(to_batch=0), dict(table=None), dict(held=None), dict(free=None),
               dict(count=None), dict(new_table=None), dict(new_held=None), dict(new_free=None), dict(new_count=None), dict(parents=None),
               dict(lens=None), dict(status=None),
               # overlaps: the target on the source, on the call's inputs, on itself, on the cache; the scratch; the cache's own
               dict(new_table=4 * A), dict(new_table=4 * A + 116), dict(new_held=5 * A + 8), dict(new_free=6 * A + 156),
               dict(new_count=7 * A), dict(new_held=12 * A), dict(new_table=13 * A + 16), dict(new_held=8 * A + 196), dict(new_free=9 * A),
               dict(new_count=10 * A + 40), dict(new_table=2 * A + 64), dict(new_free=3 * A), dict(status=11 * A), dict(status=14 * A + 16),
               dict(ws=4 * A), dict(ws=12 * A), dict(ws=2 * A), dict(ws=8 * A), dict(table=2 * A + 4096), dict(parents=3 * A),
               dict(cache=_cache(ptd, v=2 * A + 64))):
        assert call(**kw) == ptd.INVALID_ARG, kw
    for kw in (dict(ws=None), dict(nbytes=need - 1), dict(ws=14 * A + 8)):
        assert call(**kw) == ptd.WORKSPACE, kw
    for kw in (dict(batch=8193), dict(to_batch=8193), dict(cache=_cache(ptd, page=24)), dict(cache=_cache(ptd, num_pages=1 << 28)),
               dict(batch=4096, cache=_cache(ptd, max_pages=1 << 20))):
        assert call(**kw) == ptd.UNSUPPORTED, kw


@pytest.mark.parametrize("name", list(COUNTS))
def test_native_calls_leave_other_arguments_alone(lib, name):
    """Host tensors, plain objects and wrong counts are not taken (None: nothing was enqueued)."""
    import torch

    from paper_2607_10661_gb300 import ptd

    f = getattr(ptd._native(), name)
    host = torch.zeros((2, 4), dtype=torch.int32)
    for filler in (host, None, 3, [1, 2], 0.5):
        assert f(*([filler] * COUNTS[name])) is None
    assert f() is None and f(*([host] * (COUNTS[name] + 1))) is None


def test_native_calls_keep_to_the_current_device(lib):
    """Tensors of another device than the current one, or of several, are left to the path that changes the device or
    raises (the calls that are taken here end at the library's own checks)."""
    import torch

    from paper_2607_10661_gb300 import ptd

    class Holder:
        def __init__(self, c, **kw):
            self.c = c
            for k, v in kw.items():
                setattr(self, k, v)

    def fakes(device):
        class Fake:
            is_cuda = True

            def __init__(self, shape, dtype=torch.int32, on=device):
                self.shape, self.dtype, self.on = tuple(shape), dtype, on
                self.nbytes = (2 if dtype == torch.bfloat16 else 4)
                for s in shape:
                    self.nbytes *= s

            def is_contiguous(self):
                return True

            def data_ptr(self):
                return A

            def stride(self):
                s, at = [], 1
                for x in reversed(self.shape):
                    s.insert(0, at)
                    at *= x
                return tuple(s)

            def get_device(self):
                return self.on

        return Fake

    BF, F = torch.bfloat16, torch.float32
    try:
        for here, current, stray in ((0, 0, None), (1, 1, None), (1, 0, None), (0, 0, 0), (0, 0, 1), (0, 0, 2), (0, 0, 3), (0, 0, 4)):
            Fake = fakes(here)
            calls = ptd._native()
            calls.load(ptd.LIB_PATH, Fake, torch.int32, F, BF, lambda d: 0, lambda: current)
            on = lambda i: 1 - here if stray == i else here
            taken = here == current and stray is None
            want = -ptd.INVALID_ARG if taken else None   # (every pointer is the same: an overlap)
            i10 = lambda i: Fake((10,), on=on(i))
            vec = Fake((10,), F)
            assert calls.token_logprobs(Fake((10, 50), BF, on(0)), i10(1), vec, Fake((10,), F, on(2)), Fake((10, 2), on=on(3)),
                                        Fake((10, 2), F), Fake((1,), on=on(4)), 1.0, 0) == want
            assert calls.lm_head_logprobs(Fake((10, 64), BF, on(0)), Fake((50, 64), BF, on(1)), i10(2), vec, None, None, None,
                                          Fake((1000,), F, on(3)), Fake((1,), on=on(4)), 1.0, 0) == want
            paged = Holder(_cache(ptd), k=Fake((1, 1), BF, on(0)), block_table=Fake((5, 10)))
            sets = [Holder(ptd._PageSet(5, A, A, A, A), sizes=(10, 40, on(1) if j else here)) for j in range(2)]
            assert calls.page_fork(paged, *sets, Fake((5,), on=on(2)), Fake((5,)), Fake((1000,), F, on(3)), Fake((1,), on=on(4)), 0) == want
            prompt = Holder(ptd._Prompt(5, 10, 8, 100, A, A))
            rows, w = Fake((10, 8, 128), BF), Fake((128,), BF)
            assert calls.prompt_norm_rope_append(prompt, Holder(_cache(ptd), k=Fake((1, 1), BF, on(0)), block_table=Fake((5, 10))), 0,
                                                 i10(1), i10(9), Fake((10, 8, 128), BF, on(2)), rows, rows, rows, Fake((128,), BF, on(3)),
                                                 w, 1e-6, 1e4, Fake((1,), on=on(4)), 0) == want
            tree = Holder(ptd._Tree(5, 10, 8, 100, A, A, A), ctx_lens=Fake((5,), on=on(1)))
            q = Fake((2, 10, 8, 128), BF)
            assert calls.tree_norm_rope_append(tree, paged, 0, Fake((2, 10, 8, 128), BF, on(2)), q, q, q, Fake((2, 128), BF, on(3)),
                                               Fake((2, 128), BF), 1e-6, 1e4, Fake((1,), on=on(4)), None, 0) == want
    finally:
        ptd._calls = None
        ptd._native()


def test_binding_refuses_sets_of_another_cache(lib, monkeypatch):
    import types

    from paper_2607_10661_gb300 import ptd

    class Refuse:
        def __getattr__(self, name):
            return lambda *a: None

    monkeypatch.setattr(ptd, "_calls", Refuse())
    cache = types.SimpleNamespace(c=_cache(ptd), page_size=16)
    good = types.SimpleNamespace(sizes=(10, 40, 0), c=ptd._PageSet(3, A, A, A, A))
    for bad in ((11, 40, 0), (10, 41, 0)):
        other = types.SimpleNamespace(sizes=bad, c=good.c)
        for pair in ((good, other), (other, good)):
            with pytest.raises(ValueError, match="page set"):
                ptd.page_fork(cache, *pair, None, None, None, None)
            with pytest.raises(ValueError, match="page set"):
                ptd.page_fork_workspace_size(cache, *pair)
    cache.page_size = 0
    with pytest.raises(ValueError, match="page set"):
        ptd.page_fork_workspace_size(cache, good, good)


def test_trees_beyond_the_cache_are_refused(monkeypatch):
    import types

    import torch

    from paper_2607_10661_gb300 import ptd

    tree = types.SimpleNamespace(batch=3, total_nodes=5)
    q = torch.zeros((2, 5, 4, 16))
    for cache in (types.SimpleNamespace(sequences=2, page_size=16), types.SimpleNamespace(sequences=4, page_size=0)):
        cache.head_dim, cache.k, cache.num_kv_heads = 16, q, 4
        with pytest.raises(ValueError, match="sequences"):
            ptd.tree_norm_rope_append(tree, cache, 0, q, q, q, q, q, q, 1e-6, 1e4, None)
    with pytest.raises(ValueError, match="layers"):
        ptd.tree_norm_rope_append(tree, cache, 0, q[0], q, q, q, q, q, 1e-6, 1e4, None)


def test_oracle_forks_by_hand():
    """Pages of 16.  Sequence 0 has 36 positions in pages 4, 2, 6, sequence 1 20 in 4, 1 (page 4 shared), sequence 2 has
    page 7.  Two targets go on from sequence 0 (the first keeps page 6), one from its first 20 (page 2 is somebody's full
    page: copied), one from sequence 1; sequence 2 ends."""
    table = [[4, 2, 6, -1], [4, 1, -1, -1], [7, -1, -1, -1]]
    rows, free, copies = oracle.page_fork(table, [3, 2, 1], [0, 3, 5], [1, 0, 0, 0, -1], [20, 36, 36, 20, 9], 16)
    assert rows == [[4, 1], [4, 2, 6], [4, 2, 5], [4, 3], []] and free == [0, 7] and copies == [(6, 5, 4), (2, 3, 4)]
    # everything ends: the shared page comes back once
    assert oracle.page_fork(table, [3, 2, 1], [0], [-1], [0], 16) == ([[]], [0, 4, 2, 6, 1, 7], [])
    # cut to a page's end: nothing is copied, nothing kept by itself
    assert oracle.page_fork(table, [3, 2, 1], [], [0, 0], [32, 16], 16) == ([[4, 2], [4]], [6, 1, 7], [])
    assert oracle.page_fork(table, [3, 2, 1], [], [0, 0], [36, 36], 16) is None


def test_oracle_log_probabilities_by_hand():
    lp, ent, idx, val = oracle.token_logprobs([[0.0, 0.0, -np.inf, 0.0], [math.log(4), 0.0, 0.0, -np.inf], [-np.inf] * 4],
                                              [1, 0, 2], 1.0, 3)
    assert np.allclose(lp[:2], [-math.log(3), math.log(4 / 6)]) and lp[2] == -np.inf
    assert np.allclose(ent, [math.log(3), -(4 / 6) * math.log(4 / 6) + 2 * (1 / 6) * math.log(6), 0.0])
    assert idx.tolist() == [[0, 1, 3], [0, 1, 2], [0, 1, 2]] and np.allclose(val[1], np.log([4 / 6, 1 / 6, 1 / 6]))
    lp, ent, _, _ = oracle.token_logprobs([[2.0, 4.0]], [-1], 2.0, 0)
    assert lp[0] == -np.inf and np.allclose(ent, oracle.token_logprobs([[1.0, 2.0]], [0], 1.0, 0)[1])


def test_oracle_head_norm():
    """A head of equal values has norm |x|: +-1 times the weight, then the rotation; the mean square of any other is 1."""
    x = np.array([[[3.0, 3.0, -3.0, -3.0], [1.0, 2.0, 3.0, 4.0]]])
    w = np.array([1.0, 2.0, 3.0, 4.0])
    assert np.allclose(oracle.head_norm_rope(x, w, [0], 10.0, 0.0)[0, 0], [1.0, 2.0, -3.0, -4.0])
    assert np.allclose((oracle.head_norm_rope(x, np.ones(4), [7], 10.0, 0.0) ** 2).mean(-1), 1.0)
    assert np.allclose(oracle.head_norm_rope(x, w, [7], 10.0, 0.0), oracle.rope(oracle.head_norm_rope(x, w, [0], 10.0, 0.0), [7], 10.0))


def test_sizes_beyond_32_bits_are_not_cut_off(lib, monkeypatch):
    """A size or a layer that the library takes in 32 bits is refused where it has more, not taken modulo 2^32."""
    import contextlib
    import types

    import torch

    from paper_2607_10661_gb300 import ptd

    class Refuse:
        def __getattr__(self, name):
            return lambda *a: None

    monkeypatch.setattr(ptd, "_calls", Refuse())
    monkeypatch.setattr(ptd, "_dev", lambda t, name, dtype=None, row_strided=False: None if t is None else A)
    monkeypatch.setattr(ptd, "_one_device", lambda *t: contextlib.nullcontext())
    far = 1 << 32
    meta = lambda *shape, dtype=torch.bfloat16: torch.empty(shape, dtype=dtype, device="meta")
    i32, f32 = (lambda *s: meta(*s, dtype=torch.int32)), (lambda *s: meta(*s, dtype=torch.float32))
    refused = pytest.raises(ctypes.ArgumentError, match="32 bits")
    with refused:
        ptd.token_logprobs(meta(1, far + 5), i32(1), f32(1), None, None, None, i32(1), stream=0)
    with refused:
        ptd.lm_head_logprobs(meta(2, 64), meta(far + 5, 64), i32(2), f32(2), None, None, None, meta(8), i32(1), stream=0)
    with refused:
        ptd.lm_head_logprobs(meta(2, far + 64), meta(5, far + 64), i32(2), f32(2), None, None, None, meta(8), i32(1), stream=0)
    with refused:
        ptd.lm_head_logprobs(meta(far + 2, 64), meta(5, 64), i32(far + 2), f32(far + 2), None, None, None, meta(8), i32(1), stream=0)
    for sizes in ((far + 5, 100, 1), (5, far + 100, 1), (5, 100, far)):
        with refused:
            ptd.lm_head_logprobs_workspace_size(*sizes)
    cache = types.SimpleNamespace(c=_cache(ptd), k=meta(2, 40, 16, 8, 128), head_dim=128, num_kv_heads=8, sequences=2, page_size=16)
    tree = types.SimpleNamespace(c=ptd._Tree(2, 20, 16, 100, A, A, A), batch=2, total_nodes=20, ctx_lens=None)
    q, kv, w = meta(2, 20, 32, 128), meta(2, 20, 8, 128), meta(2, 128)
    with refused:
        ptd.tree_norm_rope_append(tree, cache, far, q, kv, kv, q, w, w, 1e-6, 1e4, i32(1), stream=0)
    wide = meta(1, 20, far + 32, 128)
    with refused:
        ptd.tree_norm_rope_append(tree, cache, 0, wide, kv[:1], kv[:1], wide, w[:1], w[:1], 1e-6, 1e4, i32(1), stream=0)
    monkeypatch.setattr(ptd, "_batch_of_cache", lambda *a: None)
    monkeypatch.setattr(ptd, "_rows3", lambda t, name, dt, n, heads, d: (A, t.stride(0), t.shape[1]))
    prompt = types.SimpleNamespace(c=ptd._Prompt(2, 20, 8, 100, A, A), total_tokens=20)
    with refused:
        ptd.prompt_norm_rope_append(prompt, cache, far + 1, i32(20), i32(20), q[0], kv[0], kv[0], q[0], w[0], w[0], 1e-6, 1e4, i32(1),
                                    stream=0)
