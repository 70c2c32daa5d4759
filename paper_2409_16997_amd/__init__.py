"""INT-FlashAttention forward for AMD MI355X: thin Python binding over the C ABI of libintfa.so.

Every step of the path runs in the hand-written HIP kernels of csrc/; this package only marshals
arguments (torch is used for device memory and streams).  There is no CPU fallback: if the library
has not been built, loading it raises.
"""
from .binding import (  # noqa: F401
    IFA_F32, IFA_F16, IFA_BF16, IntfaError, lib, lib_path, quantize_tokenwise, quantize_headwise, quantize_blockwise, quantize_qk, quantize_qkv,
    int_flash_attn_fwd, int_flash_attn_fwd_splitk, splitk_workspace_bytes, block_cols, int_flash_attn_fwd_half, block_cols_half, debug_fwd, status_str,
    int_flash_attn_fwd_window, window_workspace_bytes, int_flash_attn_fwd_prefix, prefix_workspace_bytes, key_weights, key_weights_workspace_bytes, evict_keys,
    append_keys, read_keys, int_flash_attn_fwd_int4, int4_workspace_bytes, IFA_CACHE_I8_F16, IFA_CACHE_I8, IFA_CACHE_I4,
)
