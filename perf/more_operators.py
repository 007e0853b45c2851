"""What the operators of a training step around a decoder's blocks are timed on and compared with.

The attention and MLP blocks of the library begin behind the norm of the hidden state and end with gradients.  Six
operators stand in front of them, between them and behind them:

``emb``       embedding_fwd: rows of the table for the tokens of a call, times a factor, in bf16.
``emb_bwd``   embedding_bwd: the table's gradient, the sum of the rows of dy that belong to each token id.
``ln``        layernorm_fwd: layer norm of the hidden state, which a block's output is added to first.
``ln_bwd``    layernorm_bwd: its gradients, the one that reaches the hidden state beside the norm added to dx.
``rms_bwd``   rmsnorm_bwd: the same for the RMS norm.
``clip``      clip_grads: the norm over all gradients of a step, and the gradients scaled down to a given norm, to new
              tensors or in place.

A table may be one of several shards (`shards`) that hold `vocab` rows each: tokens of the other shards have rows of
zeros and no gradient.  How often a token occurs goes as the inverse of its rank, as in text: one id has 6 % of all
tokens.  The hidden sizes are those of the 8B- and 32B-class layers of jet_inputs.py and generic ones, token counts run
from one to the 16384 of the training workloads, twice that for the table's gradient.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

BF16, F32, F64 = torch.bfloat16, torch.float32, torch.float64
EPS = 1e-5
LAYER_8B, LAYER_32B = (4096, 1024, 14336), (5120, 1024, 27648)     # hidden, keys' and values' columns, columns of the MLP


def _emb(name, kind, tokens, hidden, vocab, shards, f32):
    return dict(name=name, kind=kind, tokens=tokens, hidden=hidden, vocab=vocab, shards=shards, f32=f32)


def _norm(name, kind, tokens, hidden, res):
    return dict(name=name, kind=kind, tokens=tokens, hidden=hidden, res=res)


def _clip(name, layers, sizes, vocab, ratio, inplace):
    return dict(name=name, kind="clip", layers=layers, hidden=sizes[0], kv=sizes[1], inter=sizes[2], vocab=vocab, ratio=ratio,
                inplace=inplace)


def listed():
    return [
        # a decode step of the last answer of a rollout batch
        _emb("emb_1_8b", "emb", 1, 4096, 131072, 1, False),
        # forward of a training step of the 32B class from the table's f32 masters
        _emb("emb_16384_32b", "emb", 16384, 5120, 131072, 1, True),
        # a short ragged batch of a small model
        _emb("emb_bwd_1001_1k", "emb_bwd", 1001, 1024, 32001, 1, True),
        # the whole table's gradient of a training step of the 8B class
        _emb("emb_bwd_16384_8b", "emb_bwd", 16384, 4096, 131072, 1, True),
        # one of eight shards of the table, with twice as many tokens
        _emb("emb_bwd_32768_32b_shard", "emb_bwd", 32768, 5120, 16384, 8, False),
        # a decode step: one row and the output of the block in front of it
        _norm("ln_1_8b", "ln", 1, 4096, True),
        # forward of a training step
        _norm("ln_16384_8b", "ln", 16384, 4096, True),
        # gradient of a short ragged batch of a small model, at its last norm
        _norm("ln_bwd_1001_2k", "ln_bwd", 1001, 2048, False),
        # gradients of training steps
        _norm("ln_bwd_16384_8b", "ln_bwd", 16384, 4096, True),
        _norm("rms_bwd_16384_32b", "rms_bwd", 16384, 5120, True),
        # a small model whose gradients are within the limit
        _clip("clip_small", 6, (512, 128, 1536), 8191, 2.0, True),
        # layers of the 8B class and the table, gradients too large
        _clip("clip_8b", 2, LAYER_8B, 131072, 0.7, False),
    ]


def _spread(rng, low, high):
    """A whole number whose logarithm is uniform over [low, high]."""
    return min(high, max(low, int(math.exp(rng.uniform(math.log(low), math.log(high + 1))))))


def draw(rng):
    kind = rng.choice(["emb", "emb_bwd", "emb_bwd", "ln", "ln_bwd", "rms_bwd", "clip"])
    most = max(work(c)["bytes"] for c in listed() if c["kind"] == kind)
    case = None
    while case is None or work(case)["bytes"] > most:
        hidden = rng.choice([LAYER_8B[0], LAYER_32B[0], 8 * _spread(rng, 8, 1024), 8 * _spread(rng, 8, 1024)])
        if kind in ("emb", "emb_bwd"):
            case = _emb("", kind, _spread(rng, 1, 16384 if kind == "emb" else 32768), hidden, _spread(rng, 1000, 131072),
                        rng.choice([1, 1, 2, 8]), rng.random() < 0.5)
        elif kind == "clip":
            sizes = rng.choice([LAYER_8B, LAYER_32B, (hidden, 64 * rng.randint(1, 16), 8 * _spread(rng, 16, 2048))])
            ratio = rng.choice([0.1, 0.6, 2.0, 10.0])
            case = _clip("", rng.randint(1, 6), sizes, _spread(rng, 1000, 131072), ratio, ratio > 1 and rng.random() < 0.5)
        else:
            case = _norm("", kind, _spread(rng, 1, 16384), hidden, rng.random() < 0.6)
    del case["name"]
    return case


# ------------------------------------------------------------------ inputs

def _normal(gen, shape, std=1.0, dtype=BF16):
    return torch.randn(shape, generator=gen, device="cuda").mul_(std).to(dtype)


def _hidden_state(gen, T, H):
    """Some channels far larger than the others, and a mean."""
    x = torch.randn((T, H), generator=gen, device="cuda").add_(0.1)
    x[:, torch.randperm(H, generator=gen, device="cuda")[:-(-H // 100)]] *= 50.0
    return x.to(BF16)


def _gradient_shapes(case):
    """(shape, dtype) of a step's gradients: each layer's four matrices in bf16 and four norms' weights in f32, the last norm's, the table's."""
    H, kv, I = case["hidden"], case["kv"], case["inter"]
    layer = [((H + 2 * kv, H), BF16), ((H, H), BF16), ((2 * I, H), BF16), ((H, I), BF16), ((128,), F32), ((128,), F32), ((H,), F32), ((H,), F32)]
    return layer * case["layers"] + [((H,), F32), ((case["vocab"], H), BF16)]


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    kind = case["kind"]
    s = dict(kind=kind)
    if kind == "clip":
        s["grads"] = [_normal(gen, shape, 1e-3, dtype) for shape, dtype in _gradient_shapes(case)]
        s["max_norm"] = case["ratio"] * 1e-3 * math.sqrt(sum(g.numel() for g in s["grads"]))
        s["out"] = None if case["inplace"] else [torch.empty_like(g) for g in s["grads"]]
        return s
    T, H = case["tokens"], case["hidden"]
    if kind in ("emb", "emb_bwd"):
        V, n = case["vocab"], case["vocab"] * case["shards"]
        rank = torch.rand((T,), generator=gen, device="cuda", dtype=F64).mul_(math.log(n + 1)).exp_().long().sub_(1).clamp_(0, n - 1)
        s["ids"] = torch.randperm(n, generator=gen, device="cuda")[rank]
        s["first"] = case["shards"] // 2 * V
        s["rows"], s["scale"], s["dtype"] = V, math.sqrt(H), F32 if case["f32"] else BF16
        if kind == "emb":
            s["w"] = _normal(gen, (V, H), 0.02, s["dtype"])
        else:
            s["dy"] = _normal(gen, (T, H), 1e-3)
        return s
    s["x"] = _hidden_state(gen, T, H)
    s["gamma"] = (1.0 + 0.2 * torch.randn((H,), generator=gen, device="cuda")).to(BF16)
    if kind == "ln":
        s["beta"] = _normal(gen, (H,), 0.1)
        s["res"] = _normal(gen, (T, H)) if case["res"] else None
    else:
        s["dy"] = _normal(gen, (T, H), 1e-3)
        s["res"] = _normal(gen, (T, H), 1e-3) if case["res"] else None
    return s


# ------------------------------------------------------------- plain forms

def _in_shard(s):
    """Rows of the table that the tokens have, and which of them it holds."""
    row = s["ids"] - s["first"]
    here = (row >= 0) & (row < s["rows"])
    return row.clamp(0, s["rows"] - 1), here


def _plain_emb(s):
    row, here = _in_shard(s)
    return (s["w"][row].float() * s["scale"]).masked_fill(~here[:, None], 0).to(BF16)


def _plain_emb_bwd(s):
    row, here = _in_shard(s)
    dw = torch.zeros((s["rows"], s["dy"].shape[1]), dtype=F32, device="cuda")
    return dw.index_add_(0, row, s["dy"].float().masked_fill(~here[:, None], 0)).mul_(s["scale"]).to(s["dtype"])


def _plain_ln(s):
    out = {}
    x = s["x"].float()
    if s["res"] is not None:
        out["sum"] = (x + s["res"].float()).to(BF16)
        x = out["sum"].float()
    d = x - x.mean(dim=1, keepdim=True)
    r = torch.rsqrt((d * d).mean(dim=1, keepdim=True) + EPS)
    out["y"] = (d * r * s["gamma"].float() + s["beta"].float()).to(BF16)
    return out


def _plain_norm_bwd(s):
    x, dy = s["x"].float(), s["dy"].float()
    layer = s["kind"] == "ln_bwd"
    d = x - x.mean(dim=1, keepdim=True) if layer else x
    r = torch.rsqrt((d * d).mean(dim=1, keepdim=True) + EPS)
    n = d * r
    g = dy * s["gamma"].float()
    dx = g - n * (g * n).mean(dim=1, keepdim=True)
    if layer:
        dx = dx - g.mean(dim=1, keepdim=True)
    dx = dx * r
    if s["res"] is not None:
        dx = dx + s["res"].float()
    sums = ((dy * n).sum(dim=0), dy.sum(dim=0))
    return (dx.to(BF16), *(sums if layer else sums[:1]))


def _plain_clip(s):
    norm = torch.stack([g.float().square().sum(dtype=F64) for g in s["grads"]]).sum().sqrt()
    factor = torch.where(norm.isfinite() & (norm > s["max_norm"]), s["max_norm"] / norm, torch.ones_like(norm)).float()
    to = s["grads"] if s["out"] is None else s["out"]
    return (norm.float(), *[o.copy_(g.float() * factor) for o, g in zip(to, s["grads"])])


def _own(s):
    import paper_2601_14243_amd as jet
    kind = s["kind"]
    if kind == "emb":
        return jet.embedding_fwd(s["ids"], s["w"], s["scale"], first=s["first"])
    if kind == "emb_bwd":
        return jet.embedding_bwd(s["ids"], s["dy"], s["rows"], s["scale"], first=s["first"], dtype=s["dtype"])
    if kind == "ln":
        return jet.layernorm_fwd(s["x"], s["gamma"], s["beta"], EPS, residual=s["res"])
    if kind == "ln_bwd":
        return jet.layernorm_bwd(s["dy"], s["x"], s["gamma"], EPS, dres=s["res"])
    if kind == "rms_bwd":
        return jet.rmsnorm_bwd(s["dy"], s["x"], s["gamma"], EPS, dres=s["res"])
    norm = jet.clip_grads(s["grads"], s["max_norm"], out=s["out"])
    return (norm, *(s["grads"] if s["out"] is None else s["out"]))


def run(state):
    if own:
        return _own(state)
    return {"emb": _plain_emb, "emb_bwd": _plain_emb_bwd, "ln": _plain_ln, "ln_bwd": _plain_norm_bwd, "rms_bwd": _plain_norm_bwd,
            "clip": _plain_clip}[state["kind"]](state)


# ---------------------------------------------------- the definition, 64 bits

def _exact_emb(s):
    y = torch.zeros((s["ids"].shape[0], s["w"].shape[1]), dtype=F64, device="cuda")
    for t, i in enumerate((s["ids"] - s["first"]).tolist()):
        if 0 <= i < s["rows"]:
            y[t] = s["w"][i]
    return y * s["scale"]


def _exact_emb_bwd(s):
    """Token by token in the order of the ids: every sum is one of consecutive rows."""
    ids, order = torch.sort(s["ids"] - s["first"])
    keep = (ids >= 0) & (ids < s["rows"])
    ids, order = ids[keep], order[keep]
    present, counts = torch.unique_consecutive(ids, return_counts=True)
    dw = torch.zeros((s["rows"], s["dy"].shape[1]), dtype=F64, device="cuda")
    at = 0
    for i, n in zip(present.tolist(), counts.tolist()):
        dw[i] = s["dy"][order[at:at + n]].to(F64).sum(dim=0)
        at += n
    return dw * s["scale"]


def _exact_ln(s):
    x = s["x"].to(F64)
    out = {}
    if s["res"] is not None:
        out["sum"] = x + s["res"].to(F64)
        x = out["sum"].to(BF16).to(F64)                          # the norm is that of the hidden state as it is kept
    var, mean = torch.var_mean(x, dim=1, unbiased=False, keepdim=True)
    out["y"] = (x - mean) / torch.sqrt(var + EPS) * s["gamma"].to(F64) + s["beta"].to(F64)
    return out


def _exact_norm_bwd(s):
    """Derivatives with respect to the mean and the mean square, and through them."""
    x, dy = s["x"].to(F64), s["dy"].to(F64)
    H = x.shape[1]
    layer = s["kind"] == "ln_bwd"
    c = x - x.sum(dim=1, keepdim=True) / H if layer else x
    std = torch.sqrt(c.square().sum(dim=1, keepdim=True) / H + EPS)
    dn = dy * s["gamma"].to(F64)
    d_std = -(dn * c).sum(dim=1, keepdim=True) / std.square()
    dc = dn / std + d_std * c / (H * std)
    if layer:
        dc = dc - dc.sum(dim=1, keepdim=True) / H
    if s["res"] is not None:
        dc = dc + s["res"].to(F64)
    return (dc, (dy * (c / std)).sum(dim=0), *([dy.sum(dim=0)] if layer else []))


def _exact_clip(s):
    norm = math.sqrt(sum(float(torch.linalg.vector_norm(g, dtype=F64)) ** 2 for g in s["grads"]))
    factor = s["max_norm"] / norm if norm > s["max_norm"] else 1.0
    return (norm, *[g.to(F64) * factor for g in s["grads"]])


def exact(case, seed):
    s = prepare(case, seed)
    return {"emb": _exact_emb, "emb_bwd": _exact_emb_bwd, "ln": _exact_ln, "ln_bwd": _exact_norm_bwd, "rms_bwd": _exact_norm_bwd,
            "clip": _exact_clip}[case["kind"]](s)


# --------------------------------------------------------------------- work

def _distinct(tokens, n):
    """How many of n ids `tokens` tokens have, on average."""
    r = np.arange(1, n + 1, dtype=np.float64)
    return float(-np.expm1(tokens * np.log1p(-np.log1p(1 / r) / math.log(n + 1.0))).sum())


def work(case):
    kind, H = case["kind"], case["hidden"]
    if kind == "clip":
        sizes = [(math.prod(shape), 2 if dtype is BF16 else 4) for shape, dtype in _gradient_shapes(case)]
        return {"bytes": (1 if case["inplace"] else 2) * sum(n * b for n, b in sizes), "flops": 3 * sum(n for n, _ in sizes)}
    T = case["tokens"]
    if kind in ("emb", "emb_bwd"):
        V, shards, size = case["vocab"], case["shards"], 4 if case["f32"] else 2
        if kind == "emb":
            return {"bytes": 8 * T + 2 * T * H + size * H * _distinct(T, V * shards) / shards, "flops": T * H}
        return {"bytes": 8 * T + 2 * T * H / shards + size * V * H, "flops": T * H / shards}
    if kind == "ln":
        return {"bytes": (8 if case["res"] else 4) * T * H, "flops": 8 * T * H}
    return {"bytes": (8 if case["res"] else 6) * T * H, "flops": 14 * T * H}
