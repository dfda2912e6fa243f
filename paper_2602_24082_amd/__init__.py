"""Preference-packing hot path for AMD MI355X (gfx950).

The computation lives in libppattn.so (HIP kernels + host planner, C ABI in
include/pp_attn.h); `binding` marshals torch tensors into it, `workload` draws
seeded synthetic packed batches.
"""
from .binding import (Cache, PPError, make_cache, pp_attn_bwd, pp_attn_fwd, pp_cache_accept, pp_cache_append,  # noqa: F401
                      pp_cache_compact, pp_cache_fork, pp_cache_free, pp_cache_reserve, pp_cache_shared,
                      pp_cross_attn_bwd, pp_cross_attn_fwd, pp_dpo_loss, pp_pack_export, pp_policy_loss, pp_seq_logprob,
                      pp_timing_enable, pp_timing_get, pp_timing_reset, pp_tok_logprob, pp_tok_logprob_bwd,
                      pp_tok_logprob_bwd_rows, pp_tree_attn_fwd, pp_verify_draft, pp_workspace_size)
from .workload import BY_NAME, CONFIGS, Enc, Pack, config_pack, make_enc, make_pack  # noqa: F401

__version__ = "0.1.0"
