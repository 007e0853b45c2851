"""Composition of the library's entry points into the attention block of a decoder layer, beside mlp_block.py: FP8 linear layers with
FP8-saved activations around the attention operators, which run in bf16.  The rollout calls (prefill, decode) and the training forward
pass go through the same projections and the same norm and rotation, so that a token gets the same queries, keys and values in both, to the
bit.  Its attention is the same within roundings only: decode sums in another order than the forward pass, and that goes by the sizes of
the batch, so what lies behind it (o, y and the layers above) may differ in the last bits between rollout and training.

Every arithmetic step is one call into libjet.so; this module only orders the calls and keeps the saved tensors.  Layout: the q, k and v
projections are one weight [(n_q + 2 n_kv) dim, H] (query heads, key heads, value heads), so their output is one tensor; the values stay
in it, and their gradient goes to the same columns of the gradient that the projection's backward pass consumes.

    forward :  x --row quant--> (qx)  --FProp W_qkv-->  qkv  --norm, rotation-->  q, k  --attention-->  o, lse
               o --row quant--> (qo)  --FProp W_o-->  y
    saved   :  qx, qo (FP8 + scales), qkv, q, k, o (bf16), lse (f32)
    backward:  dy --row+col quant--> DGrad W_o^T --> do ;  WGrad(dy^T, qo^T) --> dW_o
               attention backward --> dq, dk, dv ;  norm and rotation backward --> dqkv, dgamma
               dqkv --row+col quant--> DGrad W_qkv^T --> dx ;  WGrad(dqkv^T, qx^T) --> dW_qkv
"""
from __future__ import annotations

import torch

from . import binding as jet


class AttentionWeights:
    """FP8 copies of the two master weights, (q, s, qT, sT) each, and the norm weights of the heads (or None)."""

    def __init__(self, w_qkv, w_o, n_q: int, n_kv: int, gamma_q=None, gamma_k=None, eps: float = 1e-6):
        self.n_q, self.n_kv, self.hidden = n_q, n_kv, w_qkv.shape[1]
        self.dim = w_qkv.shape[0] // (n_q + 2 * n_kv)
        if w_qkv.shape[0] != (n_q + 2 * n_kv) * self.dim or tuple(w_o.shape) != (self.hidden, n_q * self.dim):
            raise ValueError("w_qkv must be [(n_q + 2 n_kv) dim, hidden] and w_o [hidden, n_q dim]")
        self.qkv = jet.quant_weight(w_qkv, transposed=True)
        self.o = jet.quant_weight(w_o, transposed=True)
        self.gamma_q, self.gamma_k, self.eps = gamma_q, gamma_k, eps


def angle_table(positions: int, dim: int, base: float = 1e6, device="cuda"):
    """The table that qk_norm_rope takes: f32 [positions, dim], cosines of a position's angles, then their sines (formed in 64 bits)."""
    inv = base ** (-torch.arange(0, dim, 2, dtype=torch.float64, device=device) / dim)
    ang = torch.arange(positions, dtype=torch.float64, device=device)[:, None] * inv
    return torch.cat([ang.cos(), ang.sin()], dim=1).float()


def _heads(x, w: AttentionWeights, table, positions, cache=None, slots=None):
    """x -> its FP8 pair, the projection's output, and the rotated queries and keys."""
    qx = jet.quant_act(x)
    qkv = jet.fp8_linear_fwd(qx["q_row"], qx["s_row"], w.qkv[0], w.qkv[1])
    q, k = jet.qk_norm_rope(qkv, w.n_q, w.n_kv, table, positions, w.gamma_q, w.gamma_k, w.eps, cache, slots)
    return qx, qkv, q, k


def _project(o, w: AttentionWeights):
    qo = jet.quant_act(o.view(o.shape[0], w.n_q * w.dim))
    return qo, jet.fp8_linear_fwd(qo["q_row"], qo["s_row"], w.o[0], w.o[1])


def forward(x, w: AttentionWeights, table, positions, cu, cache=None, slots=None):
    """x bf16 [M, H] of packed sequences (rows cu[s] .. cu[s + 1] - 1, int32) -> (y bf16 [M, H], saved).  With a cache the keys and
    values also go to their slots: prefill."""
    qx, qkv, q, k = _heads(x, w, table, positions, cache, slots)
    v = qkv.view(-1, w.n_q + 2 * w.n_kv, w.dim)[:, w.n_q + w.n_kv:]
    o, lse = jet.attention_fwd(q, k, v, cu_q=cu)
    qo, y = _project(o, w)
    return y, {"qx": qx, "qkv": qkv, "q": q, "k": k, "v": v, "o": o, "lse": lse, "qo": qo, "table": table, "positions": positions, "cu": cu}


def decode(x, w: AttentionWeights, table, positions, cache, slots, pages, lengths):
    """One token per sequence, x bf16 [B, H]: its key and value go to their slots, and it attends over the first lengths[b] rows of its
    pages, itself among them.  Returns y bf16 [B, H]."""
    _, _, q, _ = _heads(x, w, table, positions, cache, slots)
    return _project(jet.attention_decode(q, cache, pages, lengths), w)[1]


def backward(saved, dy, w: AttentionWeights):
    """dy bf16 [M, H], M a multiple of 128 -> dict(dx, dw_qkv, dw_o in bf16, dgamma_q, dgamma_k in f32 or None), plus the intermediate
    tensors (for tests)."""
    s = saved
    M, rotated = dy.shape[0], w.n_q + w.n_kv
    qdy = jet.quant_act(dy, row=True, col=True)
    do = jet.fp8_linear_dgrad(qdy["q_row"], qdy["s_row"], w.o[2], w.o[3])
    qoT = jet.quant_act(s["qo"]["q_row"], s["qo"]["s_row"], row=False, col=True)
    dw_o = jet.fp8_linear_wgrad(qdy["q_colT"], qdy["s_colT"], qoT["q_colT"], qoT["s_colT"])
    dqkv = torch.empty_like(s["qkv"])
    dq, dk = torch.empty_like(s["q"]), torch.empty_like(s["k"])
    dv = dqkv.view(M, -1, w.dim)[:, rotated:]
    jet.attention_bwd(s["q"], s["k"], s["v"], s["o"], s["lse"], do.view(M, w.n_q, w.dim), cu_q=s["cu"], out=(dq, dk, dv))
    _, dgamma_q, dgamma_k = jet.qk_norm_rope_bwd(dq, dk, s["qkv"], s["table"], s["positions"], w.gamma_q, w.gamma_k, w.eps, out=dqkv)
    qd = jet.quant_act(dqkv, row=True, col=True)
    dx = jet.fp8_linear_dgrad(qd["q_row"], qd["s_row"], w.qkv[2], w.qkv[3])
    qxT = jet.quant_act(s["qx"]["q_row"], s["qx"]["s_row"], row=False, col=True)
    dw_qkv = jet.fp8_linear_wgrad(qd["q_colT"], qd["s_colT"], qxT["q_colT"], qxT["s_colT"])
    return {"dx": dx, "dw_qkv": dw_qkv, "dw_o": dw_o, "dgamma_q": dgamma_q, "dgamma_k": dgamma_k, "do": do, "dq": dq, "dk": dk, "dqkv": dqkv}
