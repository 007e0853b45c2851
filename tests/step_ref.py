"""The operators of a training step around the blocks (embedding, layer and RMS norm, gradient norm and clipping) in 64 bits, each with a bound
on how far an implementation may be off that works in binary32 and rounds its results once.  A bf16 rounding is off by at most BF of
its value, one of binary32 by at most F; a sum of n terms by at most (n + 1) F of the sum of their magnitudes, whatever the order.
1.01 stands for products of such terms."""
from __future__ import annotations

import math

import torch

BF = torch.finfo(torch.bfloat16).eps / 2
F = torch.finfo(torch.float32).eps / 2
F64 = torch.float64
LEAST = {torch.bfloat16: 2.0 ** -134, torch.float32: 2.0 ** -150}       # half the smallest subnormal
STEP = {torch.bfloat16: BF, torch.float32: F}


def in_shard(ids, first, rows):
    row = ids.long() - first
    return row.clamp(0, rows - 1), (row >= 0) & (row < rows)


def embedding(ids, w, scale, first):
    row, here = in_shard(ids, first, w.shape[0])
    y = (w.double()[row] * scale).masked_fill(~here[:, None], 0)
    return y, y.abs() * (BF + F) * 1.01 + LEAST[torch.bfloat16]           # one product, then bf16


def embedding_backward(ids, dy, rows, scale, first, dtype, base=None):
    row, here = in_shard(ids, first, rows)
    d = dy.double().masked_fill(~here[:, None], 0)
    zero = torch.zeros((rows, dy.shape[1]), dtype=F64, device=dy.device)
    n = here.double()[:, None]
    if len(ids) > 50000:                                                  # on the GPU, additions to one row wait for each other
        zero, row, d, n = zero.cpu(), row.cpu(), d.cpu(), n.cpu()
    dw, mag = ((zero.index_add(0, row, v) * s).to(dy.device) for v, s in ((d, scale), (d.abs(), abs(scale))))
    n = zero[:, :1].index_add(0, row, n).to(dy.device)
    off = (n + 2) * F * mag                                               # the sum and its product with the scale
    if base is not None:
        dw = dw + base.double()
        off = off + F * dw.abs()
    return dw, (off + STEP[dtype] * dw.abs()) * 1.01 + LEAST[dtype]


ADD = 44 * F       # of a row's sum in which no value passes through more than 43 additions: 32 columns of a lane, then lanes and waves in pairs


def _normalized(x, eps, layer):
    """n = (x - mean) r (RMS: x r), 1 / sqrt(.), bounds on the former and on the latter's relative error.  The sum under the root, 1 / K and the
    product with it, the root and the quotient; for n a subtraction, a product and the mean, which is corrected by the mean of the
    differences from it, so that it is off by the error of that sum alone."""
    mean = lambda v: v.mean(dim=1, keepdim=True)
    d = x - mean(x) if layer else x
    r, r_off = 1 / (mean(d * d) + eps).sqrt(), (ADD + 2 * F) / 2 + 2 * F
    n = d * r
    off_mean = ADD * mean(n.abs()) if layer else 0 * mean(n)
    return n, r, n.abs() * (2 * F + r_off) + off_mean, r_off, off_mean


def layer_norm(x, gamma, beta, eps):
    n, _, off_n, _, _ = _normalized(x.double(), eps, True)
    y = n * gamma.double() + (0 if beta is None else beta.double())
    return y, (off_n * gamma.double().abs() + y.abs() * (BF + F)) * 1.01 + LEAST[torch.bfloat16]


def norm_backward(dy, x, gamma, eps, dres, layer):
    """dx, dgamma, dbeta (RMS: None) and bounds on them."""
    dy, gamma, x = dy.double(), gamma.double(), x.double()
    mean = lambda v: v.mean(dim=1, keepdim=True)
    n, r, off_n, r_off, off_mean = _normalized(x, eps, layer)
    g = dy * gamma
    c1 = mean(g * n)
    c2 = mean(g) if layer else torch.zeros_like(c1)
    t = r * (g - c2 - n * c1)
    dx = t + (0 if dres is None else dres.double())
    off_c1 = (ADD + 2 * F) * mean((g * n).abs()) + off_mean * c2.abs() + (3 * F + r_off) * c1.abs()
    off_c2 = (ADD + F) * mean(g.abs()) + 2 * F * c2.abs() if layer else 0 * c1
    off = F * (g.abs() + c2.abs()) + off_c2 + off_n * c1.abs() + n.abs() * off_c1 + 2 * F * (g - c2 - n * c1).abs()
    dx_off = (r * off + (r_off + F) * t.abs() + (BF + F) * dx.abs()) * 1.01 + LEAST[torch.bfloat16]
    M = dy.shape[0]
    dgamma, dbeta = (dy * n).sum(dim=0), dy.sum(dim=0)
    dg_off = (dy.abs() * (off_n + (M + 2) * F * n.abs())).sum(dim=0) * 1.01 + F * dgamma.abs() + LEAST[torch.float32]
    db_off = (M + 2) * F * dy.abs().sum(dim=0) * 1.01 + LEAST[torch.float32]
    return (dx, dgamma, dbeta if layer else None), (dx_off, dg_off, db_off)


def norm(tensors):
    return math.sqrt(sum(float(t.double().square().sum()) for t in tensors))


def clipped(tensors, max_norm, given=None):
    """The tensors scaled down, and bounds: the norm is right to a few 2^-53 (or given), the factor rounded, the product, the result's type."""
    total = norm(tensors) if given is None else given
    f = max_norm / total if math.isfinite(total) and total > max_norm else 1.0
    want = [t.double() * f for t in tensors]
    return want, [w.abs() * (0 if f == 1.0 else (STEP[t.dtype] + 2 * F) * 1.01) + (0 if f == 1.0 else LEAST[t.dtype]) for w, t in zip(want, tensors)]


def check(got, want, tol, name):
    got = got.double()
    bad = ~((got - want).abs() <= tol)
    if bad.any():
        i = tuple(int(v[0]) for v in bad.nonzero(as_tuple=True))
        worst = ((got - want).abs() / tol.clamp(min=1e-300)).nan_to_num(nan=math.inf).max().item()
        raise AssertionError(f"{name}: {int(bad.sum())} of {bad.numel()} outside, worst {worst:.3g} bounds; at {i}: {got[i].item()!r}, "
                             f"want {want[i].item()!r} +- {tol[i].item():.3g}")
