"""Norms with the append of tokens with many heads (more than a CTA takes at once, or keeps in shared memory), and the LM head's
alternatives of random values against the exact ones.  Tolerances as in test_gpu_forks.py."""
import pytest
import torch

import test_gpu_forks as forks
from paper_2607_10661_gb300 import ptd

pytestmark = pytest.mark.gpu
DEV = "cuda"
BF16, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module", autouse=True)
def _built():
    import __graft_entry__

    __graft_entry__.build()


# (pairs of 16-byte vectors of a token: 640, 448, 768, 1536, 1280, 385, and heads of no power of two: element by element)
WIDE = [(BF16, 64, 8, 128, 16, True), (BF16, 40, 8, 128, 0, False), (BF16, 32, 32, 128, 16, False), (F32, 32, 32, 128, 16, True),
        (BF16, 64, 8, 256, 0, True), (BF16, 375, 5, 16, 16, True), (BF16, 96, 32, 96, 16, False)]


@pytest.mark.parametrize("tokens", [1, 37, 700])   # (by many threads a token, then by few)
@pytest.mark.parametrize("case", WIDE, ids=str)
def test_prompt_norms_of_many_heads(case, tokens):
    forks.test_prompt_norm_rope_append(*case, tokens)


# (bytes of a layer's rows and tables: 51200, 51200, 102400 and 43520, over the 43008 that a CTA takes, so element by element;
# 34816 and 43008: one layer a CTA)
@pytest.mark.parametrize("nodes,layers", [([1], 1), ([63], 5), ([7, 128, 1, 33], 2)])
@pytest.mark.parametrize("case", [(BF16, 64, 64, 128, 16, True), (F32, 32, 32, 128, 0, True), (BF16, 64, 64, 256, 16, True),
                                  (BF16, 144, 9, 128, 0, True),
                                  (BF16, 64, 32, 128, 16, True), (BF16, 128, 16, 128, 0, True)], ids=str)
def test_tree_norms_of_many_heads(case, nodes, layers):
    forks.test_tree_norm_rope_append(*case, nodes, layers)


@pytest.mark.parametrize("rows,vocab,d,k,T", [(200, 3001, 1024, 4, 1.5), (63, 32000, 2048, 16, 1.0), (300, 5000, 512, 8, 0.7),
                                              (1100, 2000, 64, 16, 1.0)])
def test_lm_head_alternatives_of_random_values(rows, vocab, d, k, T):
    """A logit is off by a = d 2^-23 sum |h w| at most, so the j-th largest is off by a too: the values come in order, and each is
    within the tolerance of the exact one in its place."""
    g = torch.Generator(device=DEV).manual_seed(rows)
    h = torch.randn((rows, d), generator=g, device=DEV).to(BF16)
    w = (torch.randn((vocab, d), generator=g, device=DEV) * 4 / d ** 0.5).to(BF16)
    tokens = torch.randint(0, vocab, (rows,), generator=g, device=DEV).to(torch.int32)
    out, status = forks._outputs(rows, k), torch.zeros(1, dtype=torch.int32, device=DEV)
    ws = torch.empty(ptd.lm_head_logprobs_workspace_size(rows, vocab, k), dtype=torch.uint8, device=DEV)
    ptd.lm_head_logprobs(h, w, tokens, *out, ws, status, T)
    accurate = d * 2.0 ** -23 * float((h.double().abs() @ w.double().abs().t()).max())
    logits = h.double() @ w.double().t()
    forks._check_logprobs(logits, tokens, T, k, *out, accurate=accurate)
    assert status.item() == 0
    val = out[3]
    assert (val[:, 1:] <= val[:, :-1]).all()
    z = logits / T
    exact = torch.log_softmax(z, -1).topk(k).values
    tol = z.abs().amax(-1)[:, None] * 2.0 ** -21 + (vocab / 256 + 64) * 2.0 ** -24 + 2 * accurate / T + exact.abs() * 2.0 ** -21
    assert ((val.double() - exact).abs() <= tol).all()
