"""MI355X (gfx950) implementation of FQ-ViT's integer hot path: PTF LayerNorm
and Log-Int-Softmax attention with BitShift Attn x V, the linear layers,
rotary positions and requantization around them, and the step over a stream of
tokens (RMS norm, paged cache, attention over it, eviction from it).

The computation lives in libfqvit.so (HIP kernels behind the C ABI of
include/fqvit.h); this package only builds and binds it.
"""
from .binding import (FqError, activation_table, codes_ld,  # noqa: F401
                      linear_fold_int8, linear_int8, linear_int32,
                      lis_attention_head, lis_attention_qk,
                      lis_attn_v_shift, lis_attn_v_shift_wide,
                      lis_softmax_log4, ptf_calibrate, ptf_calibrate_noalloc,
                      ptf_calibrate_workspace_bytes,
                      ptf_layernorm_int8, ptf_quantize_int8, requant_dyadic_int8, requant_heads_int8,
                      rope_qkv_int8, rope_table_int16, status_str,
                      time_next_call,
                      version)
from .decode import (kv_cache_append_int8, kv_cache_evict, lis_attention_paged,  # noqa: F401
                     lis_attention_paged_workspace_bytes, rmsnorm_int8, rmsnorm_rows_int8)

__all__ = ["ptf_layernorm_int8", "lis_softmax_log4", "lis_attn_v_shift", "lis_attn_v_shift_wide",
           "lis_attention_head",
           "lis_attention_qk",
           "ptf_calibrate", "ptf_calibrate_noalloc", "ptf_calibrate_workspace_bytes",
           "ptf_quantize_int8",
           "requant_dyadic_int8", "requant_heads_int8",
           "linear_fold_int8", "linear_int8", "linear_int32", "activation_table",
           "rope_table_int16", "rope_qkv_int8",
           "rmsnorm_int8", "rmsnorm_rows_int8", "kv_cache_append_int8", "lis_attention_paged",
           "lis_attention_paged_workspace_bytes", "kv_cache_evict",
           "FqError", "codes_ld", "status_str", "time_next_call",
           "version"]
