"""MI355X-native static-tree relaxed verification (LANTERN++ hot path).

The product is ``liblpp.so`` (hand-written HIP for gfx950, C ABI in
``include/lpp.h``); this package is its thin ctypes binding.
"""
from .binding import (  # noqa: F401
    LIB_PATH, LPP_BF16, LPP_F32, LPP_OK, LPP_EINVAL, LPP_EUNSUPPORTED, LPP_ENOWORKSPACE, LPP_EHIP,
    LppError, Tree, lib,
    lpp_build_neighbours, lpp_build_neighbours_workspace,
    lpp_tree_attention, lpp_tree_attention_gqa, lpp_tree_attention_workspace,
    lpp_tree_attention_layers, lpp_tree_attention_layers_workspace,
    lpp_relaxed_verify, lpp_relaxed_verify_workspace, lpp_relaxed_verify_additive, lpp_relaxed_verify_static,
    lpp_commit_kv, lpp_probe_stream_read, lpp_relaxed_verify_sampled, lpp_relaxed_verify_opts,
    LPP_BOUND_MULTIPLICATIVE, LPP_BOUND_ADDITIVE, LPP_RULE_PREFIX, LPP_RULE_SKIP,
    LPP_SIBLINGS_IID, LPP_SIBLINGS_DISTINCT,
    PagedCache, lpp_paged_commit_kv, lpp_paged_append_kv,
    lpp_paged_tree_attention, lpp_paged_chunk_attention, lpp_paged_attention_workspace,
    Rotary, lpp_rotary_qkv, LPP_ROTARY_HALF, LPP_ROTARY_INTERLEAVED,
    LPP_ROTARY_NONE, LPP_ROTARY_LINEAR, LPP_ROTARY_NTK, LPP_ROTARY_YARN,
    lpp_adjust_logits, lpp_token_counts, lpp_commit_counts,
)
