"""MI355X-native A2SF hot path: masked attention fused with forgotten-score bookkeeping and
budgeted KV-cache eviction (arxiv 2407.20485), and the operators of a decoder layer around it (norm, 8-bit products,
rotary positions, sampling), and a cache in pages that evicts nothing.  All compute runs in liba2sf.so (HIP, gfx950)
behind the C ABI of include/a2sf.h; `binding` marshals arguments, `synth` draws workloads."""
from .binding import (A2SF_BF16, A2SF_EVICT_FAST, A2SF_EVICT_STABLE, A2SF_F32, A2SF_MAX_CAPACITY,
                      A2SFError, Cache, a2sf_compact, a2sf_decode_step, a2sf_prefill, a2sf_select,
                      a2sf_status_string, a2sf_workspace_bytes, a2sf_prefill_alpha_per_head,
                      a2sf_decode_step_alpha_per_head, a2sf_ideal_similarity,
                      a2sf_decode_step_static_ws, A2SF_STATIC_WS_BYTES, a2sf_similarity_mean,
                      a2sf_decode_plan, a2sf_prefill_windowed, a2sf_prefill_chunk,
                      a2sf_prefill_gqa, a2sf_decode_step_gqa, a2sf_prefill_chunk_gqa,
                      A2SF_MAX_ROTARY_PARTS, A2SF_MAX_ROW, A2SF_MAX_VOCABULARY, A2SF_WIDE_SUMS, a2sf_matmul_scaled,
                      a2sf_matmul_workspace_bytes, a2sf_quantize, a2sf_quantize_weight, a2sf_rms_norm, a2sf_rotary,
                      a2sf_rotary_table, a2sf_sample,
                      A2SF_E4M3, A2SF_MAX_ALTERNATIVES, A2SF_NO_WINDOW, Pages, a2sf_log_probs, a2sf_paged_append,
                      a2sf_paged_attention, a2sf_paged_workspace_bytes)

__all__ = ["A2SF_BF16", "A2SF_F32", "A2SF_EVICT_FAST", "A2SF_EVICT_STABLE", "A2SF_MAX_CAPACITY",
           "A2SFError", "Cache", "a2sf_compact", "a2sf_decode_step", "a2sf_prefill", "a2sf_select",
           "a2sf_status_string", "a2sf_workspace_bytes", "a2sf_prefill_alpha_per_head",
           "a2sf_decode_step_alpha_per_head", "a2sf_ideal_similarity", "a2sf_decode_step_static_ws",
           "A2SF_STATIC_WS_BYTES", "a2sf_similarity_mean", "a2sf_decode_plan", "a2sf_prefill_windowed", "a2sf_prefill_chunk",
           "a2sf_prefill_gqa", "a2sf_decode_step_gqa", "a2sf_prefill_chunk_gqa",
           "A2SF_MAX_ROTARY_PARTS", "A2SF_MAX_ROW", "A2SF_MAX_VOCABULARY", "A2SF_WIDE_SUMS", "a2sf_matmul_scaled",
           "a2sf_matmul_workspace_bytes", "a2sf_quantize", "a2sf_quantize_weight", "a2sf_rms_norm", "a2sf_rotary",
           "a2sf_rotary_table", "a2sf_sample", "A2SF_E4M3", "A2SF_MAX_ALTERNATIVES", "A2SF_NO_WINDOW", "Pages", "a2sf_log_probs",
           "a2sf_paged_append", "a2sf_paged_attention", "a2sf_paged_workspace_bytes"]
