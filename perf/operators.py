"""What the attention operators of the library are timed on and compared with.

Five operators of a decoder layer stand between the q/k/v projection and the output projection:

``qk``      qk_norm_rope: norm of every query and key head and the rotation of its pairs of channels by the
            token's position, from the projection's output [T, (n_q + 2 n_kv) D]; with `page` > 0 the rotated
            keys and the values also go to their slots of a paged cache, as serving does.
``qk_bwd``  its gradient with respect to the projection's output and to the two norm weights.
``fwd``     attention_fwd: causal attention of packed sequences with shared key/value heads, with the
            logarithm of each row's sum of exponentials.
``bwd``     attention_bwd: gradients of q, k and v from saved q, k, v, output and logarithms.
``decode``  attention_decode: one query token per sequence against a paged cache in bf16, or in E4M3 with a
            scale for each token and head.

The head counts are those of the 8B- and 32B-class layers of jet_inputs.py (4096 / 128 = 32 and 5120 / 128 = 40
query heads, 1024 / 128 = 8 key/value heads) and of smaller generic layers with 64 channels per head.  Lengths run
from a single token to 16384, the token count of the training workloads.
"""
from __future__ import annotations

import math
import random

import torch

own = False

POSITIONS = 32768          # rows of the table of angles
ROPE_BASE = 1.0e6
EPS = 1e-6
BF16, F32, F64 = torch.bfloat16, torch.float32, torch.float64
CHUNK = 1 << 28            # scores that the plain form and the definition hold at a time


def _qk(name, tokens, n_q, n_kv, dim, norm, page):
    return dict(name=name, kind="qk", tokens=tokens, n_q=n_q, n_kv=n_kv, dim=dim, norm=norm, page=page)


def _qk_bwd(name, tokens, n_q, n_kv, dim, norm):
    return dict(name=name, kind="qk_bwd", tokens=tokens, n_q=n_q, n_kv=n_kv, dim=dim, norm=norm)


def _attention(name, kind, seqs, shortest, longest, prefix, n_q, n_kv, dim, lens_seed=0):
    return dict(name=name, kind=kind, seqs=seqs, shortest=shortest, longest=longest, prefix=prefix, n_q=n_q,
                n_kv=n_kv, dim=dim, lens_seed=lens_seed)


def _decode(name, seqs, shortest, longest, n_q, n_kv, dim, page, fp8, lens_seed=0):
    return dict(name=name, kind="decode", seqs=seqs, shortest=shortest, longest=longest, n_q=n_q, n_kv=n_kv, dim=dim,
                page=page, fp8=fp8, lens_seed=lens_seed)


def listed():
    return [
        # the last answer of a rollout batch: one token, its key and value go to the cache
        _qk("qk_token_8b", 1, 32, 8, 128, True, 64),
        # forward of a training step, 16384 tokens
        _qk("qk_16384_8b", 16384, 32, 8, 128, True, 0),
        # gradient of a short ragged batch of a small model
        _qk_bwd("qk_bwd_1001_d64", 1001, 16, 2, 64, True),
        # gradient of a training step of the 32B class
        _qk_bwd("qk_bwd_16384_32b", 16384, 40, 8, 128, True),
        # prefill of one short prompt
        _attention("fwd_37_8b", "fwd", 1, 37, 37, 0, 32, 8, 128),
        # log-probs of a batch of answers of very different lengths
        _attention("fwd_packed_32b", "fwd", 24, 60, 4096, 0, 40, 8, 128, 1),
        # the longest sequence
        _attention("fwd_16384_8b", "fwd", 1, 16384, 16384, 0, 32, 8, 128),
        # actor update on answers of very different lengths
        _attention("bwd_packed_8b", "bwd", 24, 60, 4096, 0, 32, 8, 128, 2),
        # actor update on one long answer
        _attention("bwd_8192_8b", "bwd", 1, 8192, 8192, 0, 32, 8, 128),
        # decode of the last answer of a rollout batch
        _decode("decode_1x700_8b", 1, 700, 700, 32, 8, 128, 64, False),
        # a decode step of a rollout batch, answers between 500 and 8192 tokens
        _decode("decode_64x8k_8b", 64, 500, 8192, 32, 8, 128, 64, False, 3),
        # the same of the 32B class with long answers and the cache in E4M3
        _decode("decode_128x16k_32b_fp8", 128, 1000, 16384, 40, 8, 128, 64, True, 4),
    ]


def _spread(rng, low, high):
    """A whole number whose logarithm is uniform over [low, high]."""
    return min(high, max(low, int(math.exp(rng.uniform(math.log(low), math.log(high + 1))))))


def draw(rng):
    kind = rng.choice(["qk", "qk_bwd", "fwd", "fwd", "bwd", "bwd", "decode", "decode"])
    n_q, n_kv, dim = rng.choice([(32, 8, 128), (40, 8, 128), (16, 2, 64), (8, 8, 64), (12, 2, 128), (6, 1, 64)])
    if kind == "qk":
        case = _qk("", _spread(rng, 1, 16384), n_q, n_kv, dim, rng.random() < 0.7, rng.choice([0, 16, 64]))
    elif kind == "qk_bwd":
        case = _qk_bwd("", _spread(rng, 1, 16384), n_q, n_kv, dim, rng.random() < 0.7)
    elif kind == "decode":
        case = None
        while case is None or work(case)["bytes"] > work(listed()[-1])["bytes"]:
            longest = _spread(rng, 1, 16384)
            case = _decode("", _spread(rng, 1, 128), _spread(rng, 1, longest), longest, n_q, n_kv, dim,
                           rng.choice([16, 32, 64, 128]), rng.random() < 0.5, rng.randrange(1 << 20))
    else:
        most = max(work(c)["flops"] for c in listed() if c["kind"] == kind)
        case = None
        while case is None or work(case)["flops"] > most:
            longest = _spread(rng, 1, 16384 if kind == "fwd" else 8192)
            case = _attention("", kind, _spread(rng, 1, 24), _spread(rng, 1, longest), longest,
                              rng.choice([0, 0, _spread(rng, 1, 2048)]), n_q, n_kv, dim, rng.randrange(1 << 20))
    del case["name"]
    return case


def _lengths(case):
    """Lengths of the sequences: log-uniform, the first one the longest."""
    rng = random.Random(case["lens_seed"])
    return [case["longest"]] + [_spread(rng, case["shortest"], case["longest"]) for _ in range(case["seqs"] - 1)]


def _spans(lengths):
    """Prefix sums with a leading zero."""
    out = [0]
    for n in lengths:
        out.append(out[-1] + n)
    return out


# ------------------------------------------------------------------ inputs

def _normal(gen, shape, std=1.0):
    return torch.randn(shape, generator=gen, device="cuda").mul_(std).to(BF16)


def _table(dim):
    """[POSITIONS, dim] f32: cosines of a position's angles, then their sines; angles in 64 bits."""
    inv = ROPE_BASE ** (-torch.arange(0, dim, 2, dtype=F64, device="cuda") / dim)
    ang = torch.arange(POSITIONS, dtype=F64, device="cuda")[:, None] * inv
    return torch.cat([ang.cos(), ang.sin()], dim=1).to(F32)


def _prepare_qk(case, gen):
    T, n_q, n_kv, dim = case["tokens"], case["n_q"], case["n_kv"], case["dim"]
    s = dict(n_q=n_q, n_kv=n_kv, dim=dim, table=_table(dim))
    s["qkv"] = _normal(gen, (T, (n_q + 2 * n_kv) * dim), 1.5)
    if case["kind"] == "qk" and case["page"]:                        # serving: every token of another sequence
        s["positions"] = torch.randint(0, POSITIONS, (T,), generator=gen, device="cuda", dtype=torch.int32)
    else:                                                            # packed answers of up to 4096 tokens
        s["positions"] = (torch.arange(T, device="cuda", dtype=torch.int32) + 1234) % 4096
    for name in ("gamma_q", "gamma_k"):
        s[name] = (1.0 + 0.2 * torch.randn((dim,), generator=gen, device="cuda")).to(BF16) if case["norm"] else None
    if case["kind"] == "qk_bwd":
        s["dq"] = _normal(gen, (T, n_q, dim), 1e-3)
        s["dk"] = _normal(gen, (T, n_kv, dim), 1e-3)
    elif case["page"]:
        n_pages = T // case["page"] + 9
        shape = (n_pages, n_kv, case["page"], dim)
        s["cache_k"], s["cache_v"] = _normal(gen, shape), _normal(gen, shape)
        s["slots"] = torch.randperm(n_pages * case["page"], generator=gen, device="cuda")[:T].contiguous()
    return s


def _prepare_attention(case, gen):
    lens_q = _lengths(case)
    lens_k = [n + case["prefix"] for n in lens_q]
    cu_q, cu_k = _spans(lens_q), _spans(lens_k)
    n_q, n_kv, dim = case["n_q"], case["n_kv"], case["dim"]
    s = dict(lens_q=lens_q, lens_k=lens_k, n_q=n_q, n_kv=n_kv, dim=dim, scale=dim ** -0.5)
    s["cu_q"] = torch.tensor(cu_q, dtype=torch.int32, device="cuda")
    s["cu_k"] = torch.tensor(cu_k, dtype=torch.int32, device="cuda")
    s["q"] = _normal(gen, (cu_q[-1], n_q, dim), 1.5)
    s["k"] = _normal(gen, (cu_k[-1], n_kv, dim), 1.5)
    # values stay where the projection left them: a slice of [T, (n_q + 2 n_kv) dim]
    s["v"] = _normal(gen, (cu_k[-1], n_q + 2 * n_kv, dim))[:, n_q + n_kv:]
    if case["kind"] == "bwd":
        s["o"], s["lse"] = _plain_fwd(s)                             # what the forward pass saved
        s["do"] = _normal(gen, (cu_q[-1], n_q, dim), 1e-3)
    return s


def _prepare_decode(case, gen):
    lens, page = _lengths(case), case["page"]
    n_q, n_kv, dim = case["n_q"], case["n_kv"], case["dim"]
    pages = [-(-n // page) for n in lens]
    n_pages = sum(pages) + 3
    order = torch.randperm(n_pages, generator=gen, device="cuda").to(torch.int32)
    table = torch.zeros((len(lens), max(pages)), dtype=torch.int32, device="cuda")
    at = 0
    for i, n in enumerate(pages):
        table[i, :n] = order[at:at + n]
        at += n
    s = dict(lens=lens, n_q=n_q, n_kv=n_kv, dim=dim, page=page, scale=dim ** -0.5, pages=table,
             lengths=torch.tensor(lens, dtype=torch.int32, device="cuda"), cache_k_scale=None, cache_v_scale=None)
    s["q"] = _normal(gen, (len(lens), n_q, dim), 1.5)
    for name, std in (("cache_k", 1.5), ("cache_v", 1.0)):
        shape = (n_pages, n_kv, page, dim)
        if case["fp8"]:
            x = torch.randn(shape, generator=gen, device="cuda").mul_(std)
            scale = x.abs().amax(dim=-1) / 448.0
            s[name] = (x / scale[..., None]).to(torch.float8_e4m3fn).view(torch.uint8)
            s[name + "_scale"] = scale
        else:
            s[name] = _normal(gen, shape, std)
    return s


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    kind = case["kind"]
    make = _prepare_qk if kind in ("qk", "qk_bwd") else _prepare_decode if kind == "decode" else _prepare_attention
    s = make(case, gen)
    s["kind"] = kind
    if own and "cache_k" in s:
        import paper_2601_14243_amd as jet
        s["cache"] = jet.KvCache(s["cache_k"], s["cache_v"], s.get("cache_k_scale"), s.get("cache_v_scale"))
    return s


# ------------------------------------------------------------- plain forms

def _rotate(x, cos, sin):
    """Pairs (i, i + dim / 2) of x [T, n, dim] by the angles of each token."""
    a, b = x.chunk(2, dim=-1)
    return torch.cat([a * cos - b * sin, b * cos + a * sin], dim=-1)


def _angles(s, dtype):
    half = s["dim"] // 2
    rows = s["table"][s["positions"].long()].to(dtype)[:, None, :]
    return rows[..., :half], rows[..., half:]


def _plain_qk(s):
    n_q, n_kv, dim = s["n_q"], s["n_kv"], s["dim"]
    x = s["qkv"].float().view(-1, n_q + 2 * n_kv, dim)
    cos, sin = _angles(s, F32)
    out = []
    for part, gamma in ((x[:, :n_q], s["gamma_q"]), (x[:, n_q:n_q + n_kv], s["gamma_k"])):
        if gamma is not None:
            part = part * torch.rsqrt((part * part).mean(dim=-1, keepdim=True) + EPS) * gamma.float()
        out.append(_rotate(part, cos, sin).to(BF16))
    if "slots" in s:
        page = s["cache_k"].shape[2]
        where, row = s["slots"] // page, s["slots"] % page
        s["cache_k"][where, :, row] = out[1]
        s["cache_v"][where, :, row] = x[:, n_q + n_kv:].to(BF16)
        out += [s["cache_k"], s["cache_v"]]
    return tuple(out)


def _plain_qk_bwd(s):
    n_q, n_kv, dim = s["n_q"], s["n_kv"], s["dim"]
    x = s["qkv"].float().view(-1, n_q + 2 * n_kv, dim)
    cos, sin = _angles(s, F32)
    dx, dgamma = [], []
    for part, dy, gamma in ((x[:, :n_q], s["dq"], s["gamma_q"]), (x[:, n_q:n_q + n_kv], s["dk"], s["gamma_k"])):
        g = _rotate(dy.float(), cos, -sin)
        if gamma is not None:
            r = torch.rsqrt((part * part).mean(dim=-1, keepdim=True) + EPS)
            n = part * r
            dgamma.append((g * n).sum(dim=(0, 1)))
            g = g * gamma.float()
            g = (g - n * (g * n).mean(dim=-1, keepdim=True)) * r
        dx.append(g.to(BF16))
    return (torch.cat(dx, dim=1).flatten(1), *dgamma)


def _sequences(s):
    """(rows of q, rows of k) of each sequence."""
    q0 = k0 = 0
    for n, m in zip(s["lens_q"], s["lens_k"]):
        yield slice(q0, q0 + n), slice(k0, k0 + m)
        q0, k0 = q0 + n, k0 + m


def _row_chunks(s, n, m):
    step = max(1, CHUNK // (s["n_q"] * m))
    return [(r, min(r + step, n)) for r in range(0, n, step)]


def _hidden(r0, r1, n, m):
    """True where key j lies after row i of the last n of m positions, rows r0 to r1."""
    i = torch.arange(r0, r1, device="cuda")[:, None] + (m - n)
    return torch.arange(m, device="cuda")[None, :] > i


def _heads(x, n_kv):
    """[rows, heads, dim] -> f32 [n_kv, heads / n_kv, rows, dim], the heads of a group together."""
    return x.float().permute(1, 0, 2).reshape(n_kv, -1, x.shape[0], x.shape[2])


def _plain_fwd(s):
    o = torch.empty((s["q"].shape[0], s["n_q"], s["dim"]), dtype=BF16, device="cuda")
    lse = torch.empty((s["n_q"], s["q"].shape[0]), dtype=F32, device="cuda")
    for rq, rk in _sequences(s):
        q, k, v = _heads(s["q"][rq], s["n_kv"]), _heads(s["k"][rk], s["n_kv"]), _heads(s["v"][rk], s["n_kv"])
        n, m = q.shape[2], k.shape[2]
        kT = k.transpose(2, 3).contiguous()
        for r0, r1 in _row_chunks(s, n, m):
            scores = torch.matmul(q[:, :, r0:r1] * s["scale"], kT)
            scores.masked_fill_(_hidden(r0, r1, n, m), -math.inf)
            top = scores.amax(dim=-1, keepdim=True)
            p = scores.sub_(top).exp_()
            total = p.sum(dim=-1, keepdim=True)
            rows = torch.matmul(p, v).div_(total)
            o[rq.start + r0:rq.start + r1] = rows.flatten(0, 1).permute(1, 0, 2).to(BF16)
            lse[:, rq.start + r0:rq.start + r1] = (top + total.log()).flatten(0, 1).squeeze(-1)
    return o, lse


def _plain_bwd(s):
    dq, dk, dv = (torch.empty(x.shape, dtype=BF16, device="cuda") for x in (s["q"], s["k"], s["v"]))
    for rq, rk in _sequences(s):
        n_kv = s["n_kv"]
        q, k, v = _heads(s["q"][rq], n_kv), _heads(s["k"][rk], n_kv), _heads(s["v"][rk], n_kv)
        do, lse = _heads(s["do"][rq], n_kv), s["lse"][:, rq].reshape(n_kv, -1, q.shape[2], 1)
        n, m = q.shape[2], k.shape[2]
        kT, vT = k.transpose(2, 3).contiguous(), v.transpose(2, 3).contiguous()
        sum_k, sum_v = torch.zeros_like(k), torch.zeros_like(v)
        for r0, r1 in _row_chunks(s, n, m):
            qc, dc = q[:, :, r0:r1].contiguous(), do[:, :, r0:r1].contiguous()
            p = torch.matmul(qc * s["scale"], kT).sub_(lse[:, :, r0:r1])
            p.masked_fill_(_hidden(r0, r1, n, m), -math.inf).exp_()
            sum_v += torch.matmul(p.transpose(2, 3), dc).sum(dim=1, keepdim=True)
            dp = torch.matmul(dc, vT)
            ds = p * (dp - (p * dp).sum(dim=-1, keepdim=True)) * s["scale"]
            rows = torch.matmul(ds, k)
            dq[rq.start + r0:rq.start + r1] = rows.flatten(0, 1).permute(1, 0, 2).to(BF16)
            sum_k += torch.matmul(ds.transpose(2, 3), qc).sum(dim=1, keepdim=True)
        dk[rk] = sum_k.squeeze(1).permute(1, 0, 2).to(BF16)
        dv[rk] = sum_v.squeeze(1).permute(1, 0, 2).to(BF16)
    return dq, dk, dv


def _cached(s, name, i, n):
    """The first n rows of sequence i, f32 [n_kv, n, dim]."""
    where = s["pages"][i, :-(-n // s["page"])].long()
    x = s[name][where]
    if s[name + "_scale"] is None:
        x = x.float()
    else:
        x = x.view(torch.float8_e4m3fn).float() * s[name + "_scale"][where][..., None]
    return x.permute(1, 0, 2, 3).reshape(s["n_kv"], -1, s["dim"])[:, :n]


def _plain_decode(s):
    rows = []
    for i, n in enumerate(s["lens"]):
        q = s["q"][i].float().view(s["n_kv"], -1, s["dim"]) * s["scale"]
        k, v = _cached(s, "cache_k", i, n), _cached(s, "cache_v", i, n)
        scores = torch.matmul(q, k.transpose(1, 2).contiguous())
        p = torch.exp(scores - scores.amax(dim=-1, keepdim=True))
        rows.append((torch.matmul(p, v) / p.sum(dim=-1, keepdim=True)).view(s["n_q"], s["dim"]))
    return torch.stack(rows).to(BF16)


def _own(s):
    import paper_2601_14243_amd as jet
    kind = s["kind"]
    if kind == "qk":
        out = jet.qk_norm_rope(s["qkv"], s["n_q"], s["n_kv"], s["table"], s["positions"], s["gamma_q"], s["gamma_k"],
                               EPS, cache=s.get("cache"), slots=s.get("slots"))
        return (*out, s["cache_k"], s["cache_v"]) if "slots" in s else tuple(out)
    if kind == "qk_bwd":
        dx, dgamma_q, dgamma_k = jet.qk_norm_rope_bwd(s["dq"], s["dk"], s["qkv"], s["table"], s["positions"],
                                                      s["gamma_q"], s["gamma_k"], EPS)
        return (dx,) if dgamma_q is None else (dx, dgamma_q, dgamma_k)
    if kind == "fwd":
        return jet.attention_fwd(s["q"], s["k"], s["v"], cu_q=s["cu_q"], cu_k=s["cu_k"])
    if kind == "bwd":
        return jet.attention_bwd(s["q"], s["k"], s["v"], s["o"], s["lse"], s["do"], cu_q=s["cu_q"], cu_k=s["cu_k"])
    return jet.attention_decode(s["q"], s["cache"], s["pages"], s["lengths"])


def run(state):
    if own:
        return _own(state)
    return {"qk": _plain_qk, "qk_bwd": _plain_qk_bwd, "fwd": _plain_fwd, "bwd": _plain_bwd,
            "decode": _plain_decode}[state["kind"]](state)


# ---------------------------------------------------- the definition, 64 bits

def _exact_qk(s):
    n_q, n_kv, dim = s["n_q"], s["n_kv"], s["dim"]
    half = dim // 2
    T = s["qkv"].shape[0]
    angle = s["table"].to(F64)[s["positions"].long()]
    turn = torch.complex(angle[:, :half], angle[:, half:])[:, None, :]
    heads = s["qkv"].to(F64).view(T, n_q + 2 * n_kv, dim)
    res = []
    for first, count, gamma in ((0, n_q, s["gamma_q"]), (n_q, n_kv, s["gamma_k"])):
        h = heads[:, first:first + count]
        if gamma is not None:
            h = gamma.to(F64) * h / torch.sqrt(h.square().sum(dim=2, keepdim=True) / dim + EPS)
        z = torch.complex(h[..., :half].contiguous(), h[..., half:].contiguous()) * turn
        res.append(torch.cat([z.real, z.imag], dim=2))
    if "slots" in s:
        n_pages, _, page, _ = s["cache_k"].shape
        for old, new in ((s["cache_k"], res[1]), (s["cache_v"], heads[:, n_q + n_kv:])):
            flat = old.to(F64).permute(0, 2, 1, 3).reshape(n_pages * page, n_kv, dim)
            flat.index_copy_(0, s["slots"], new)
            res.append(flat.view(n_pages, page, n_kv, dim).permute(0, 2, 1, 3).contiguous())
    return tuple(res)


def _exact_qk_bwd(s):
    n_q, n_kv, dim = s["n_q"], s["n_kv"], s["dim"]
    half = dim // 2
    T = s["qkv"].shape[0]
    angle = s["table"].to(F64)[s["positions"].long()]
    back = torch.complex(angle[:, :half], -angle[:, half:])[:, None, :]
    heads = s["qkv"].to(F64).view(T, n_q + 2 * n_kv, dim)
    grads, weights = [], []
    for first, dy, gamma in ((0, s["dq"], s["gamma_q"]), (n_q, s["dk"], s["gamma_k"])):
        d = dy.to(F64)
        z = torch.complex(d[..., :half].contiguous(), d[..., half:].contiguous()) * back
        d = torch.cat([z.real, z.imag], dim=2)
        if gamma is not None:
            x = heads[:, first:first + d.shape[1]]
            ms = x.square().sum(dim=2, keepdim=True) / dim + EPS
            weights.append((d * x / ms.sqrt()).sum(dim=1).sum(dim=0))
            d = d * gamma.to(F64)
            d = d / ms.sqrt() - x * (d * x).sum(dim=2, keepdim=True) / (dim * ms * ms.sqrt())
        grads.append(d.reshape(T, -1))
    return (torch.cat(grads, dim=1), *weights)


def _exact_attention(s, backward):
    """One head and some rows at a time, as written in a textbook: softmax(q k^T scale) v and its derivatives."""
    o = torch.zeros(s["q"].shape, dtype=F64, device="cuda")
    lse = torch.zeros((s["n_q"], s["q"].shape[0]), dtype=F64, device="cuda")
    dq, dk, dv = (torch.zeros(s[x].shape, dtype=F64, device="cuda") for x in ("q", "k", "v"))
    group = s["n_q"] // s["n_kv"]
    q0 = k0 = 0
    for n, m in zip(s["lens_q"], s["lens_k"]):
        for h in range(s["n_q"]):
            g = h // group
            q = s["q"][q0:q0 + n, h].to(F64)
            k, v = s["k"][k0:k0 + m, g].to(F64), s["v"][k0:k0 + m, g].to(F64)
            step = max(1, CHUNK // 2 // m)
            for a in range(0, n, step):
                b = min(a + step, n)
                seen = m - n + b                                      # keys that the last of these rows sees
                x = (q[a:b] @ k[:seen].T) * s["scale"]
                late = torch.arange(seen, device="cuda") > torch.arange(m - n + a, seen, device="cuda")[:, None]
                x[late] = -math.inf
                norm = torch.logsumexp(x, dim=1)
                p = torch.exp(x - norm[:, None])
                if not backward:
                    lse[h, q0 + a:q0 + b] = norm
                    o[q0 + a:q0 + b, h] = p @ v[:seen]
                    continue
                d = s["do"][q0 + a:q0 + b, h].to(F64)
                dv[k0:k0 + seen, g] += p.T @ d
                t = d @ v[:seen].T
                t = (t - (t * p).sum(dim=1, keepdim=True)) * p * s["scale"]
                dq[q0 + a:q0 + b, h] = t @ k[:seen]
                dk[k0:k0 + seen, g] += t.T @ q[a:b]
        q0, k0 = q0 + n, k0 + m
    return (dq, dk, dv) if backward else (o, lse)


def _exact_decode(s):
    out = torch.empty(s["q"].shape, dtype=F64, device="cuda")
    group = s["n_q"] // s["n_kv"]
    for i, n in enumerate(s["lens"]):
        at = torch.arange(n, device="cuda")
        where, row = s["pages"][i].long()[at // s["page"]], at % s["page"]
        kv = []
        for name in ("cache_k", "cache_v"):
            x = s[name][where, :, row]                                # [n, n_kv, dim]
            if s[name + "_scale"] is not None:
                x = x.view(torch.float8_e4m3fn).to(F32).to(F64) * s[name + "_scale"][where, :, row].to(F64)[..., None]
            kv.append(x.to(F64))
        for g in range(s["n_kv"]):
            q = s["q"][i, g * group:(g + 1) * group].to(F64)
            p = torch.softmax((q @ kv[0][:, g].T) * s["scale"], dim=1)
            out[i, g * group:(g + 1) * group] = p @ kv[1][:, g]
    return out


def exact(case, seed):
    s = prepare(case, seed)
    kind = case["kind"]
    if kind == "qk":
        return _exact_qk(s)
    if kind == "qk_bwd":
        return _exact_qk_bwd(s)
    if kind == "decode":
        return _exact_decode(s)
    return _exact_attention(s, kind == "bwd")


# --------------------------------------------------------------------- work

def work(case):
    kind, n_q, n_kv, dim = case["kind"], case["n_q"], case["n_kv"], case["dim"]
    if kind in ("qk", "qk_bwd"):
        T = case["tokens"]
        rows = 2 * T * (n_q + n_kv) * dim                             # bytes of q and k
        angles = 4 * dim * min(T, 4096) + 4 * T
        elements = T * (n_q + n_kv) * dim
        if kind == "qk":
            moved = 2 * rows + angles
            if case["page"]:                                          # values read, keys and values written once more
                moved += 3 * 2 * T * n_kv * dim + 8 * T
            return {"bytes": moved, "flops": (7 if case["norm"] else 3) * elements}
        return {"bytes": (3 if case["norm"] else 2) * rows + angles, "flops": (14 if case["norm"] else 3) * elements}
    lens = _lengths(case)
    if kind == "decode":
        tokens = sum(lens)
        each = (dim + 4) if case["fp8"] else 2 * dim
        return {"bytes": 2 * tokens * n_kv * each + 4 * len(lens) * n_q * dim + 4 * tokens // case["page"],
                "flops": 4 * tokens * n_q * dim}
    p = case["prefix"]
    pairs = sum(n * p + n * (n + 1) // 2 for n in lens)
    t_q, t_k = sum(lens), sum(lens) + p * len(lens)
    q_bytes, k_bytes, lse = 2 * t_q * n_q * dim, 2 * t_k * n_kv * dim, 4 * t_q * n_q
    if kind == "fwd":
        return {"bytes": 2 * q_bytes + 2 * k_bytes + lse, "flops": 4 * pairs * n_q * dim}
    return {"bytes": 4 * q_bytes + 4 * k_bytes + lse, "flops": 10 * pairs * n_q * dim}
