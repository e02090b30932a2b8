"""MI355X-native WKV6 prefill: HIP kernels behind a C ABI, with a thin binding."""
from .binding import (  # noqa: F401
    WKV6_DTYPE_BF16, WKV6_DTYPE_F32, Wkv6Error, load, status_string, wkv6_append_bf16, wkv6_decode_bf16,
    wkv6_decay_lora_input_bf16, wkv6_finch_c2_append_bf16, wkv6_finch_c2_decode_bf16, wkv6_finch_c2_prefill_bf16,
    wkv6_finch_c2_prefill_bf16_moments, wkv6_finch_c2_prefill_bf16_split, wkv6_finch_c2_prefill_lora_bf16, wkv6_layernorm_apply_bf16, wkv6_layernorm_finalize,
    wkv6_key_compress_bf16,
    wkv6_finch_c2_prefill_bf16_f32out, wkv6_finch_c2_prefill_bf16_strided, wkv6_prefill_bf16,
    wkv6_prefill_bf16_f32out, wkv6_prefill_bf16_recurrent, wkv6_prefill_lora_bf16, wkv6_prefill_bf16_split, wkv6_prefill_bf16_split_noalloc,
    wkv6_prefill_bf16_strided, wkv6_prefill_f32, wkv6_split_segments, wkv6_split_workspace_bytes,
    wkv6_arena_layout, wkv6_version,
    wkv6_head_decay_backward, wkv6_head_decay_backward_workspace_bytes, wkv6_head_decay_decode, wkv6_head_decay_prefill,
    wkv6_head_decay_workspace_bytes, wkv6_layernorm_backward, wkv6_layernorm_backward_workspace_bytes, wkv6_layernorm_forward,
    wkv6_selective_scan_backward, wkv6_selective_scan_backward_workspace_bytes, wkv6_selective_scan_decode, wkv6_selective_scan_prefill,
    wkv6_selective_scan_workspace_bytes, wkv6_short_conv_backward, wkv6_short_conv_backward_workspace_bytes, wkv6_short_conv_decode,
    wkv6_short_conv_prefill)
