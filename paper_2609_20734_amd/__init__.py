"""On-Demand Attention (ODA) decode-step hot path for AMD MI355X (gfx950).

The product is the C-ABI library ``liboda.so`` (include/oda.h): hand-written
HIP kernels for Local decode attention (over the paged cache, or over the
direct-ring workspace), the recall gate with its device predicate, Full
decode attention for flagged requests only, the selected-state commit, the
operators of a step of many tenants with drafted tokens (attention over shared
prefixes, adapters beside dense layers, verification and commit of drafts), those
that take prompts in (rows appended to the paged cache, their attention over it,
log probabilities of their tokens), and
the decoder layers around them (``decoder`` composes whole synthetic decode
steps from those entry points).  This package
holds its sources (``csrc/``), its build step (``build.py``), a ctypes
binding with the same entry-point names (``_lib``), the byte accounting used
to report bandwidth (``ledger``) and the synthetic workload shapes
(``workloads``).

The binding is loaded on first use of any entry point; if ``liboda.so`` has
not been built that raises ImportError (there is no fallback path).
"""
_EXPORTS = ("HEAD_MLP", "HEAD_PAPER", "OdaError", "Shape", "attn_workspace_size", "full_decode_attn",
            "gate_desc", "gate_param_count", "gate_workspace_size", "inputs", "local_decode_attn",
            "recall_gate", "lib", "prepare_local", "prepare_full", "prepare_gate", "Call", "commit_kv", "prepare_commit",
            "commit_workspace_size",
            "DENSE_PLAIN", "DENSE_SWIGLU", "dense_desc", "dense_bf16", "qk_norm_rope", "embed_bf16", "copy_rows",
            "argmax", "prepare_dense", "prepare_qk_norm_rope", "prepare_embed", "prepare_copy_rows",
            "prepare_argmax", "stream_read", "prepare_stream_read", "rms_norm_rows", "prepare_rms_norm_rows",
            "recall_gate_static", "qkv_prep", "prepare_local_qkv", "prepare_full_qkv",
            "ring_elements", "ring_fill", "local_decode_attn_ring", "commit_kv_ring", "prepare_local_ring",
            "prefix_groups", "prefix_plan_size", "prefix_workspace_size", "prefix_plan", "prefix_decode_attn",
            "prepare_prefix_plan", "prepare_prefix_decode_attn", "lora_desc", "lora_workspace_size", "dense_lora_bf16",
            "prepare_dense_lora", "verify_desc", "verify_workspace_size", "verify_drafts", "prepare_verify_drafts", "commit_drafts", "prepare_commit_drafts",
            "F32", "BF16", "MAX_AXES", "MAX_TOP", "prompt_rows", "append_desc", "append_qkv", "prepare_append_qkv",
            "prompt_plan_size", "prompt_workspace_size", "prompt_plan", "prepare_prompt_plan", "prompt_attn",
            "prepare_prompt_attn", "logprob_desc", "logprob_workspace_size", "token_logprobs", "prepare_token_logprobs")


def __getattr__(name):
    if name in _EXPORTS:
        from . import _lib
        return _lib if name == "lib" else getattr(_lib, name)
    raise AttributeError(name)
