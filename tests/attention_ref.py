"""The attention operators in 64 bits on the CPU, from their formulas, each with a bound on how far an implementation may be off
that forms sums in binary32, rounds probabilities and score gradients to bf16 before they enter a product, and rounds its
results once.  A bf16 rounding is off by at most BF of its value, one of binary32 by at most F.  Bounds are worst cases: a sum of
n terms is off by at most (n + 1) F of the sum of their magnitudes, whatever the order."""
from __future__ import annotations

import math

import torch

BF = torch.finfo(torch.bfloat16).eps / 2
F = torch.finfo(torch.float32).eps / 2
F64 = torch.float64


def visible(n, m, causal):
    """[n, m]: whether row i sees key j; the last row sees the last key."""
    if not causal:
        return torch.ones((n, m), dtype=torch.bool)
    return torch.arange(m)[None, :] <= torch.arange(n)[:, None] + (m - n)


def _scores(q, k, scale, see):
    """Scores of one head, and how far a binary32 score may be off: dim products and sums, one factor, and in the exponent the
    subtraction of a reference of at most twice the largest magnitude and the function's own rounding."""
    s = (q @ k.T) * scale
    mag = (q.abs() @ k.abs().T) * scale
    err = (q.shape[1] + 4) * F * mag + 8 * F * mag.amax(dim=1, keepdim=True).clamp(min=1) if mag.numel() else mag
    return s.masked_fill(~see, -math.inf), err.masked_fill(~see, 0)


def forward(q, k, v, scale, see):
    """One head, f64 [n, dim], [m, dim]: o, lse and bounds on their errors."""
    n, m = see.shape
    s, e = _scores(q, k, scale, see)
    some = see.any(dim=1)
    if m == 0 or not some.any():
        z = torch.zeros_like(q)
        return dict(o=z, lse=torch.full((n,), -math.inf, dtype=F64), o_tol=z, lse_tol=torch.zeros(n, dtype=F64))
    lse = torch.logsumexp(s, dim=1)
    p = torch.exp(s - lse.masked_fill(~some, 0)[:, None])
    o = p @ v
    reach = p @ v.abs()
    e_row = e.amax(dim=1) + (m + 8) * F                         # relative, of a probability or of their sum
    o_tol = reach * (BF + 2 * e_row + (m + 8) * F)[:, None] * 1.01 + BF * o.abs() * 1.01
    lse_tol = e_row * 1.01 + 4 * F * (lse.masked_fill(~some, 0).abs() + e.new_ones(n) * 8)
    return dict(o=o, lse=lse, o_tol=o_tol, lse_tol=lse_tol)


def backward(q, k, v, do, scale, see):
    """One head: gradients and bounds on their errors, with o and lse from an implementation within forward()'s bounds."""
    n, m = see.shape
    if m == 0 or n == 0:
        z = [torch.zeros_like(x) for x in (q, k, v)]
        return z, [x.clone() for x in z]
    f = forward(q, k, v, scale, see)
    s, e = _scores(q, k, scale, see)
    some = see.any(dim=1)
    p = torch.exp(s - f["lse"].masked_fill(~some, 0)[:, None])
    rel = (e.amax(dim=1) + f["lse_tol"] + 8 * F)[:, None]       # of a probability
    dp = do @ v.T
    delta = (p * dp).sum(dim=1, keepdim=True)
    ds = p * (dp - delta)
    off = (do.abs() * f["o_tol"]).sum(dim=1, keepdim=True) + (q.shape[1] + 8) * F * (do.abs() @ v.abs().T + do.abs() @ v.abs().amax(dim=0)[:, None])
    ds_tol = p * (off + (dp - delta).abs() * 2 * rel) + BF * (ds.abs() + p * off)
    sums = lambda a, b, k_terms: (a.abs() @ b.abs()) * (k_terms + 8) * F
    dq, dk, dv = ds @ k * scale, ds.T @ q * scale, p.T @ do
    dq_tol = (ds_tol @ k.abs() + sums(ds, k, m)) * scale * 1.01
    dk_tol = (ds_tol.T @ q.abs() + sums(ds.T, q, n)) * scale * 1.01
    dv_tol = (p.T * (BF + 2 * rel.T)) @ do.abs() * 1.01 + sums(p.T, do, n)
    return [dq, dk, dv], [dq_tol, dk_tol, dv_tol]               # before the results' own rounding

def peaked_backward(q, k, v, do, scale, see):
    """dq, dk of one head and bounds that leave delta = sum_j p_ij dp_ij only its binary32 errors, and dq besides what an implementation may
    leave uncorrected of a delta that was formed from a rounded o: half a step of bf16 of sum_j |ds_ij|, which is what rounding ds may come to."""
    n, m = see.shape
    f = forward(q, k, v, scale, see)
    s, e = _scores(q, k, scale, see)
    some = see.any(dim=1)
    p = torch.exp(s - f["lse"].masked_fill(~some, 0)[:, None])
    rel = (e.amax(dim=1) + f["lse_tol"] + 8 * F)[:, None]       # of a probability
    dp = do @ v.T
    ds = p * (dp - (p * dp).sum(dim=1, keepdim=True))
    total = ds.abs().sum(dim=1, keepdim=True)
    first = (do.abs() * f["o_tol"]).sum(dim=1, keepdim=True)    # what do o may be off by
    noise = (q.shape[1] + 8) * F * (do.abs() @ v.abs().T + do.abs() @ v.abs().amax(dim=0)[:, None])
    noise = noise + (2 * rel + (m + 8) * F) * (total + first)   # of ds, and of the sum that corrects delta
    out = []
    for left, transposed in ((BF / (1 - BF) * total, False), (0 * total, True)):
        off = left + noise
        ds_tol = p * off + ds.abs() * 2 * rel + BF * (ds.abs() + p * off)
        a, t, x = (ds.T, ds_tol.T, q) if transposed else (ds, ds_tol, k)
        out.append((a @ x * scale, (t @ x.abs() + (a.abs() @ x.abs()) * (a.shape[1] + 8) * F) * scale * 1.01))
    return [out[0][0], out[1][0]], [out[0][1], out[1][1]]


def spans(cu, rows):
    """(first, end) of each sequence."""
    return [(min(max(a, 0), rows), min(max(b, 0), rows)) for a, b in zip(cu[:-1], cu[1:])]


def packed_forward(q, k, v, cu_q, cu_k, scale, causal):
    """[Tq, n_q, dim], [Tk, n_kv, dim] of any type on the CPU: o, lse [n_q, Tq] and bounds."""
    q, k, v = (x.to(F64) for x in (q, k, v))
    n_q, group = q.shape[1], q.shape[1] // k.shape[1]
    o, ot = torch.zeros_like(q), torch.zeros_like(q)
    lse, lt = torch.full((n_q, q.shape[0]), -math.inf, dtype=F64), torch.zeros((n_q, q.shape[0]), dtype=F64)
    for (a, b), (c, d) in zip(spans(cu_q, q.shape[0]), spans(cu_k, k.shape[0])):
        see = visible(b - a, d - c, causal)
        for h in range(n_q):
            r = forward(q[a:b, h], k[c:d, h // group], v[c:d, h // group], scale, see)
            o[a:b, h], ot[a:b, h], lse[h, a:b], lt[h, a:b] = r["o"], r["o_tol"], r["lse"], r["lse_tol"]
    return o, lse, ot, lt


def packed_backward(q, k, v, do, cu_q, cu_k, scale, causal):
    """dq, dk, dv and bounds, the results' rounding to bf16 included."""
    q, k, v, do = (x.to(F64) for x in (q, k, v, do))
    group = q.shape[1] // k.shape[1]
    g = [torch.zeros_like(x) for x in (q, k, v)]
    t = [torch.zeros_like(x) for x in (q, k, v)]
    for (a, b), (c, d) in zip(spans(cu_q, q.shape[0]), spans(cu_k, k.shape[0])):
        see = visible(b - a, d - c, causal)
        for h in range(q.shape[1]):
            gh, th = backward(q[a:b, h], k[c:d, h // group], v[c:d, h // group], do[a:b, h], scale, see)
            for x, y in ((g, gh), (t, th)):
                x[0][a:b, h] = y[0]
                x[1][c:d, h // group] += y[1]
                x[2][c:d, h // group] += y[2]
    return g, [tol + BF * (x.abs() + tol) for x, tol in zip(g, t)]


def norm_rope(x, gamma, table, positions, eps):
    """[T, heads, dim] f64 (gamma None: no norm) and a bound that counts some 16 binary32 roundings and the result's."""
    half = x.shape[2] // 2
    if gamma is not None:
        x = x / torch.sqrt((x * x).mean(dim=2, keepdim=True) + eps) * gamma
    row = table[positions][:, None, :]
    c, s = row[..., :half], row[..., half:]
    a, b = x[..., :half], x[..., half:]
    y = torch.cat([a * c - b * s, b * c + a * s], dim=2)
    mag = torch.cat([(a * c).abs() + (b * s).abs(), (b * c).abs() + (a * s).abs()], dim=2)
    noise = (16 + x.shape[2]) * F * mag
    return y, noise + BF * (y.abs() + noise)


def norm_rope_backward(dy, x, gamma, table, positions, eps):
    """dx and its bound, dgamma [dim] (None without norm) and its bound."""
    T, heads, dim = dy.shape
    half = dim // 2
    row = table[positions][:, None, :]
    c, s = row[..., :half], row[..., half:]
    a, b = dy[..., :half], dy[..., half:]
    g = torch.cat([a * c + b * s, b * c - a * s], dim=2)
    g_mag = torch.cat([(a * c).abs() + (b * s).abs(), (b * c).abs() + (a * s).abs()], dim=2)
    if gamma is None:
        noise = 4 * F * g_mag
        return g, noise + BF * (g.abs() + noise), None, None
    r = 1 / torch.sqrt((x * x).mean(dim=2, keepdim=True) + eps)
    n = x * r
    dgamma = (g * n).sum(dim=(0, 1))
    dgamma_tol = (T * heads + dim + 24) * F * (g_mag * n.abs()).sum(dim=(0, 1))
    u, u_mag = g * gamma, g_mag * gamma.abs()
    dx = r * (u - n * (u * n).mean(dim=2, keepdim=True))
    noise = (2 * dim + 32) * F * r * (u_mag + n.abs() * (u_mag * n.abs()).mean(dim=2, keepdim=True))
    return dx, noise + BF * (dx.abs() + noise), dgamma, dgamma_tol


def cached(cache, scale, pages, n):
    """First n rows of a sequence, f64 [n, n_kv, dim]."""
    page = cache.shape[2]
    out = torch.zeros((n, cache.shape[1], cache.shape[3]), dtype=F64)
    for j in range(n):
        p, r = int(pages[j // page]), j % page
        x = cache[p, :, r]
        out[j] = x.to(F64) if scale is None else x.view(torch.float8_e4m3fn).to(torch.float32).to(F64) * scale[p, :, r].to(F64)[:, None]
    return out


def decode(q, ck, cv, ks, vs, pages, lengths, scale):
    """q [B, n_q, dim] on the CPU: o f64 and its bound."""
    o, tol = torch.zeros(q.shape, dtype=F64), torch.zeros(q.shape, dtype=F64)
    group = q.shape[1] // ck.shape[1]
    for b in range(q.shape[0]):
        n = int(lengths[b])
        if n <= 0:
            continue
        k, v = cached(ck, ks, pages[b], n), cached(cv, vs, pages[b], n)
        for h in range(q.shape[1]):
            r = forward(q[b:b + 1, h].to(F64), k[:, h // group], v[:, h // group], scale, torch.ones((1, n), dtype=torch.bool))
            o[b, h], tol[b, h] = r["o"][0], r["o_tol"][0]
    return o, tol


def check(got, want, tol, what):
    """Every element within its bound; where the bound is 0 (an empty row) the values are equal."""
    got = got.detach().cpu().to(F64)
    assert got.shape == want.shape, what
    same = (got == want) | ((got - want).abs() <= tol)
    if not same.all():
        at = tuple(int(i) for i in (~same).nonzero()[0])
        raise AssertionError(f"{what}: {int((~same).sum())} of {same.numel()} outside, first {at}: got {got[at].item()!r}, "
                             f"want {want[at].item()!r} +- {tol[at].item():.3e}")
