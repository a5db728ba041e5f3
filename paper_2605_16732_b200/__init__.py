"""DiRotQ rotation-aware W4A4 linear layer for B200: CUDA library + thin binding."""
from .binding import (  # noqa: F401
    DirotqError, Layer, alloc_workspace, dirotq_int_gemm_debug, dirotq_layer_bytes, dirotq_layer_export,
    dirotq_linear, dirotq_linear_host, dirotq_linear_noalloc, dirotq_prepare_layer, dirotq_prepare_scratch_bytes, dirotq_rotate_quantize, dirotq_w4a4_gemm,
    dirotq_workspace_bytes, dirotq_workspace_export, dirotq_workspace_status, lib,
    LAYOUT_KN, LAYOUT_NK, MX_SCALE_CEIL, MX_SCALE_FLOOR, Mxfp4, QkNorm, alloc_mxfp4_workspace, dirotq_linear_qkv, dirotq_mxfp4_alloc,
    dirotq_mxfp4_dequantize, dirotq_mxfp4_export, dirotq_mxfp4_gemm, dirotq_mxfp4_import, dirotq_mxfp4_linear, dirotq_mxfp4_qkv,
    dirotq_mxfp4_quantize, dirotq_qk_norm_rope,
)
