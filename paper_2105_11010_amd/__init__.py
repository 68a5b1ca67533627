"""SPARQ trimmed convolution-as-GEMM on AMD MI355X (gfx950).

Thin Python front end of ``libsparq.so`` (see ``include/sparq.h`` and, for the microscaled formats,
``include/sparq_mx.h`` and ``include/sparq_mx_experts.h``): the names below are the C entry points, taking torch device tensors as plain buffers.
"""
from .binding import (  # noqa: F401
    LIB_PATH, SparqConvDesc, SparqError, SparqMode, conv_desc, lib, mode, out_rows, strerror,
    sparq_conv_gemm, sparq_conv_gemm_static_ws, sparq_conv_gemm_u8, sparq_conv_plan, sparq_dequant, sparq_pack_weights, sparq_packed_bytes,
    sparq_requant, sparq_trim, sparq_workspace_bytes, sparq_packed_act_bytes, sparq_pack_act, sparq_unpack_act,
    sparq_conv_packed_workspace_bytes, sparq_conv_gemm_packed, sparq_sparse24_packed_bytes, sparq_sparse24_workspace_bytes,
    sparq_pack_weights_sparse24, sparq_conv_gemm_sparse24, sparq_sparse24_plan, sparq_set_tuning,
    sparq_mx_quantize, sparq_mx_dequantize, sparq_mx_gemm, sparq_mx_linear, sparq_mx_linear_dx, sparq_mx_linear_dw,
    sparq_mx_act, sparq_mx_act_grad, sparq_mx_norm, sparq_mx_norm_grad, sparq_mx_code_bytes, sparq_mx_scale_bytes,
    sparq_mx_gemm_workspace_bytes, sparq_mx_linear_workspace_bytes, sparq_mx_linear_dx_workspace_bytes,
    sparq_mx_linear_dw_workspace_bytes, sparq_mx_norm_grad_workspace_bytes,
    sparq_mx_sort, sparq_mx_gather, sparq_mx_combine, sparq_mx_combine_grad, sparq_mx_experts_gemm, sparq_mx_experts_linear,
    sparq_mx_experts_dx, sparq_mx_experts_dw, sparq_mx_dropout, sparq_mx_sort_workspace_bytes,
    sparq_mx_experts_gemm_workspace_bytes, sparq_mx_experts_linear_workspace_bytes, sparq_mx_experts_dx_workspace_bytes,
    sparq_mx_experts_dw_workspace_bytes,
)

__all__ = ["LIB_PATH", "SparqConvDesc", "SparqError", "SparqMode", "conv_desc", "lib", "mode", "out_rows",
           "strerror", "sparq_conv_gemm", "sparq_conv_gemm_static_ws", "sparq_conv_gemm_u8", "sparq_conv_plan", "sparq_dequant", "sparq_pack_weights",
           "sparq_packed_bytes", "sparq_requant", "sparq_trim", "sparq_workspace_bytes", "sparq_packed_act_bytes", "sparq_pack_act",
           "sparq_unpack_act", "sparq_conv_packed_workspace_bytes", "sparq_conv_gemm_packed", "sparq_sparse24_packed_bytes",
           "sparq_sparse24_workspace_bytes", "sparq_pack_weights_sparse24", "sparq_conv_gemm_sparse24", "sparq_sparse24_plan", "sparq_set_tuning",
           "sparq_mx_quantize", "sparq_mx_dequantize", "sparq_mx_gemm", "sparq_mx_linear", "sparq_mx_linear_dx",
           "sparq_mx_linear_dw", "sparq_mx_act", "sparq_mx_act_grad", "sparq_mx_norm", "sparq_mx_norm_grad",
           "sparq_mx_code_bytes", "sparq_mx_scale_bytes", "sparq_mx_gemm_workspace_bytes", "sparq_mx_linear_workspace_bytes",
           "sparq_mx_linear_dx_workspace_bytes", "sparq_mx_linear_dw_workspace_bytes", "sparq_mx_norm_grad_workspace_bytes",
           "sparq_mx_sort", "sparq_mx_gather", "sparq_mx_combine", "sparq_mx_combine_grad", "sparq_mx_experts_gemm", "sparq_mx_experts_linear",
           "sparq_mx_experts_dx", "sparq_mx_experts_dw", "sparq_mx_dropout", "sparq_mx_sort_workspace_bytes",
           "sparq_mx_experts_gemm_workspace_bytes", "sparq_mx_experts_linear_workspace_bytes", "sparq_mx_experts_dx_workspace_bytes",
           "sparq_mx_experts_dw_workspace_bytes"]
