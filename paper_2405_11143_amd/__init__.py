"""Paged decode attention for AMD MI355X (gfx950).

The rollout hot path of RLHF/RLVR training (arXiv 2405.11143): one decode
step's attention of every sequence's new query token(s) over its paged KV
cache, with grouped-query heads (also with a shared prompt prefix attended once
for all the prompt's samples), the KV-cache append before it, and the step
captured as a HIP graph, the sampled tokens' log-probabilities and entropies,
and the same step over an 8-bit KV cache with rotary positions; attention with a sliding
window, head norms with rotary positions, and block tables kept on the GPU --
hand-written HIP kernels behind a C ABI (include/).  This package is the thin Python binding of that ABI.
"""
from .pda import (EXPORTED, LIB_PATH, BoundCall, ModelStepGraph, PdaError, StepGraph, bind_append_kv, bind_decode, bind_token_logprobs,  # noqa: F401
                  load_library, make_prefix_groups,
                  make_problem, pda_append_kv, pda_decode, pda_decode_shared_prefix, pda_merge_partitions,
                  pda_partition_attention, pda_plan, pda_plan_info, pda_plan_shared_prefix, pda_prefix_groups,
                  pda_problem, pda_status_string, pda_token_logprobs, pda_validate_host, pda_workspace_bytes,
                  pda_work_order, pda_decode_reusing_order, pda_decode_noalloc, bind_decode_noalloc,
                  bind_gather_ceiling, bind_stream_ceiling,
                  pda_decode_append, bind_decode_append,
                  pda_rotary, pda_rotary_scaling, pda_rotary_inv_freq, make_rotary, pda_rotary_apply, bind_rotary_apply,
                  make_fp8_cache, pda_append_kv_fp8, bind_append_kv_fp8, pda_plan_fp8, pda_decode_fp8,
                  bind_decode_fp8, pda_read_kv_fp8, bind_read_kv_fp8,
                  pda_head_norm, pda_rotary_axes, make_head_norm, make_rotary_axes, pda_norm_rotary, bind_norm_rotary,
                  pda_norm_rotary_workspace_bytes, pda_norm_rotary_backward, bind_norm_rotary_backward,
                  pda_norm_rotary_append, bind_norm_rotary_append,
                  pda_window, pda_plan_window, pda_decode_window, bind_decode_window,
                  pda_block_pool, pda_token_rows, make_block_pool, new_block_pool, pda_blocks_resize, bind_blocks_resize,
                  pda_slot_map, bind_slot_map)
