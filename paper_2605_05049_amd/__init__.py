"""MI355X-native MoE expert layer (gfx950 HIP kernels behind a C ABI); thin ctypes binding.

Every function here only marshals arguments (torch tensors -> device pointers, current stream) and calls the
entry point of the same name declared in include/moe.h.  There is no CPU or eager fallback: if the shared
library is missing, calls raise.
"""
from .binding import (  # noqa: F401
    MoeError, Shape, abi_version, load_library, library_path, status_str, workspace_bytes, grouped_ffn_small_tiles, grouped_ffn_mid_tiles,
    moe_route_topk, moe_route_topk_bwd, moe_permute, moe_permute_noalloc, moe_permute_bwd, moe_permute_bwd_add, moe_router_fwd,
    moe_router_route_fwd,
    moe_router_bwd, moe_grouped_ffn_bwd_recompute, moe_grouped_ffn_router_bwd, moe_grouped_ffn_fwd,
    moe_grouped_ffn_bwd, moe_unpermute_combine, moe_unpermute_combine_bwd, moe_unpermute_combine_route_bwd, EXPORTED_SYMBOLS,
    profile_enable, profile_reset, profile_records, load_accumulate, load_imbalance, rebalance_experts,
    moe_halo_pack_remote, moe_halo_repack, moe_halo_unpack,
    moe_mxfp4_quantize, moe_mxfp4_quantize_t, moe_mxfp4_dequantize, moe_mxfp4_grouped_gemm, moe_mxfp4_grouped_ffn_fwd,
    mxfp4_workspace_bytes, mxfp4_grouped_gemm_large_tiles,
    FEW_TOKENS_MAX, layer_few_workspace_bytes, moe_layer_few_fwd, moe_layer_few_mxfp4_fwd,
)
from .layer import (  # noqa: F401
    MoeLayerBuffers, CapturedLayerStep, layer_forward, layer_backward, FewTokenBuffers, PromptMemory, layer_few_forward, quantize_experts,
    layer_mxfp4_forward,
)
