"""PTD tree-verify step on one GB300 (sm_103a): tree attention, per-node top-k, greedy
verification and KV compaction as hand-written CUDA kernels behind a C ABI (libptd.so).

`ptd` is the Python binding (argument marshalling only); `synthetic` draws seeded inputs.
"""
from . import ptd  # noqa: F401
from .ptd import (  # noqa: F401
    KVCache,
    PagePool,
    PageSet,
    Prompt,
    PtdError,
    StepBuffers,
    Tree,
    attention_workspace_size,
    kv_compact,
    lm_head_logprobs,
    lm_head_logprobs_workspace_size,
    page_fork,
    page_fork_workspace_size,
    prompt_attention,
    prompt_attention_workspace_size,
    prompt_norm_rope_append,
    prompt_rope_append,
    prompt_slots,
    token_logprobs,
    topk_draft,
    tree_attention,
    tree_norm_rope_append,
    tree_verify_step,
    tree_verify_step_host,
    verify_greedy,
)
