"""MI355X-native block-scaled FP8 linear layer (Jet-RL's unified precision flow), and the attention operators between
two of them.

The product is ``libjet.so`` (hand-written HIP for gfx950 behind the C ABI of
``include/jet.h``); this package is a thin binding with the same names (ctypes, and a native
extension for the tensor helpers).
PyTorch supplies device memory and streams only.
"""
from .binding import (JET_SRC_BF16, JET_SRC_FP8_ROW, JetError, fp8_linear_dgrad, fp8_linear_fwd,
                      fp8_linear_wgrad, jet_fp8_linear_dgrad, jet_fp8_linear_fwd,
                      jet_fp8_linear_wgrad, jet_quant_act, jet_quant_weight, jet_status_str,
                      jet_version, lib, quant_act, quant_weight,
                      jet_rmsnorm_quant, jet_silu_mul_quant, rmsnorm_quant, silu_mul_quant,
                      jet_silu_mul_bwd, silu_mul_bwd, jet_silu_mul_bwd_quant, silu_mul_bwd_quant,
                      KvCache, attention_bwd, attention_decode, attention_fwd, qk_norm_rope, qk_norm_rope_bwd,
                      jet_attention_bwd, jet_attention_bwd_workspace, jet_attention_decode, jet_attention_decode_workspace,
                      jet_attention_fwd, jet_qk_norm_rope, jet_qk_norm_rope_bwd, jet_qk_norm_rope_bwd_workspace,
                      JET_BF16, JET_F32, JET_I32, JET_I64, JET_NORM_LAYER, JET_NORM_RMS,
                      clip_grads, embedding_bwd, embedding_fwd, grad_norm, layernorm_bwd, layernorm_fwd, rmsnorm_bwd,
                      jet_clip_grads, jet_embedding_bwd, jet_embedding_bwd_workspace, jet_embedding_fwd, jet_grad_norm, jet_grad_norm_workspace,
                      jet_layernorm_fwd, jet_norm_bwd, jet_norm_bwd_workspace)

__all__ = [
    "JET_SRC_BF16", "JET_SRC_FP8_ROW", "JetError", "lib", "jet_version", "jet_status_str",
    "jet_quant_act", "jet_quant_weight", "jet_fp8_linear_fwd", "jet_fp8_linear_dgrad",
    "jet_fp8_linear_wgrad", "quant_act", "quant_weight", "fp8_linear_fwd", "fp8_linear_dgrad",
    "fp8_linear_wgrad", "jet_rmsnorm_quant",
    "jet_silu_mul_quant", "rmsnorm_quant", "silu_mul_quant", "jet_silu_mul_bwd", "silu_mul_bwd",
    "jet_silu_mul_bwd_quant", "silu_mul_bwd_quant",
    "KvCache", "qk_norm_rope", "qk_norm_rope_bwd", "attention_fwd", "attention_bwd", "attention_decode",
    "jet_qk_norm_rope", "jet_qk_norm_rope_bwd", "jet_qk_norm_rope_bwd_workspace", "jet_attention_fwd", "jet_attention_bwd",
    "jet_attention_bwd_workspace", "jet_attention_decode", "jet_attention_decode_workspace",
    "JET_BF16", "JET_F32", "JET_I32", "JET_I64", "JET_NORM_LAYER", "JET_NORM_RMS",
    "embedding_fwd", "embedding_bwd", "layernorm_fwd", "layernorm_bwd", "rmsnorm_bwd", "grad_norm", "clip_grads",
    "jet_embedding_fwd", "jet_embedding_bwd", "jet_embedding_bwd_workspace", "jet_layernorm_fwd", "jet_norm_bwd", "jet_norm_bwd_workspace",
    "jet_grad_norm", "jet_grad_norm_workspace", "jet_clip_grads",
]
