"""Embedding, layer and RMS norm, gradient norm and clipping on the GPU against their formulas in 64 bits (step_ref.py)."""
import math

import pytest
import torch

import step_ref as ref

pytestmark = pytest.mark.gpu
bf, f32, f64, i32, i64 = torch.bfloat16, torch.float32, torch.float64, torch.int32, torch.int64


@pytest.fixture(scope="module")
def jet():
    import paper_2601_14243_amd as j
    assert torch.cuda.is_available()
    j.lib()
    return j


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _normal(gen, shape, std=1.0, dtype=bf):
    return (torch.randn(shape, generator=gen, device="cuda") * std).to(dtype)


def _f32(x):
    return torch.tensor(x, dtype=f32).item()


def _same(a, b):
    return a.dtype == b.dtype and a.shape == b.shape and torch.equal(a.reshape(-1).view(torch.uint8), b.reshape(-1).view(torch.uint8))


# ------------------------------------------------------------------ embedding

# tokens, hidden, rows, first: one token; a row's pieces that do not fill a wave; more than one sorted block, its borders; far more tokens than rows
EMBED = [(1, 4096, 500, 0), (1, 8, 1, 0), (2, 72, 3, 0), (37, 64, 50, 7), (64, 136, 20, 0), (65, 136, 20, 0), (100, 1000, 9, -3), (1000, 520, 7001, 0),
         (1023, 8, 300, 0), (1024, 128, 5000, 0), (1025, 128, 60, 100), (3001, 264, 40, 0), (5000, 2056, 1234, 11), (9000, 24, 100000, 0), (33000, 40, 7, 0)]


def _ids(gen, T, rows, first, dtype):
    """Half of the tokens on few ids, some outside the table, padding."""
    n = rows + 5
    ids = torch.randint(0, n, (T,), generator=gen, device="cuda")
    few = torch.randint(0, min(3, rows), (T,), generator=gen, device="cuda")
    ids = torch.where(torch.rand((T,), generator=gen, device="cuda") < 0.5, few, ids) + first
    ids[torch.rand((T,), generator=gen, device="cuda") < 0.1] = first - 1
    if T == 1:
        ids[0] = first + rows - 1
    return ids.to(dtype)


@pytest.mark.parametrize("wide", [True, False])
@pytest.mark.parametrize("dtype", [bf, f32])
@pytest.mark.parametrize("T,H,V,first", EMBED)
def test_embedding_fwd(jet, T, H, V, first, dtype, wide):
    g = _gen(T + H)
    ids, w = _ids(g, T, V, first, i64 if wide else i32), _normal(g, (V, H), 0.02, dtype)
    scale = _f32(math.sqrt(H))
    y = jet.embedding_fwd(ids, w, scale, first=first)
    assert y.dtype == bf and y.shape == (T, H)
    ref.check(y, *ref.embedding(ids, w, scale, first), "y")
    out = torch.full((T, H), 7.0, dtype=bf, device="cuda")
    assert jet.embedding_fwd(ids, w, scale, first, out) is out and _same(out, y)
    one = jet.embedding_fwd(ids, w, first=first)                         # a factor of 1: the row itself, rounded
    row, here = ref.in_shard(ids, first, V)
    assert torch.equal(one, w[row].masked_fill(~here[:, None], 0).to(bf))


@pytest.mark.parametrize("dtype", [bf, f32])
@pytest.mark.parametrize("T,H,V,first", EMBED)
def test_embedding_bwd(jet, T, H, V, first, dtype):
    g = _gen(T + H + 1)
    ids, dy = _ids(g, T, V, first, i64 if T % 2 else i32), _normal(g, (T, H), 1e-3)
    scale = _f32(math.sqrt(H))
    want = ref.embedding_backward(ids, dy, V, scale, first, dtype)
    dw = jet.embedding_bwd(ids, dy, V, scale, first, dtype)
    assert dw.dtype == dtype and dw.shape == (V, H)
    ref.check(dw, *want, "dw")
    out = torch.full((V, H), float("nan"), dtype=dtype, device="cuda")   # all of it is written
    assert jet.embedding_bwd(ids, dy, V, scale, first, out=out) is out and _same(out, dw)
    base = _normal(g, (V, H), 1e-2, dtype)
    row, here = ref.in_shard(ids, first, V)
    absent = torch.ones(V, dtype=torch.bool, device="cuda")
    absent[row[here]] = False
    base[absent] = float("nan")                                          # not read, not written
    got = jet.embedding_bwd(ids, dy, V, scale, first, out=base.clone(), accumulate=True)
    assert _same(got[absent], base[absent])
    want, tol = ref.embedding_backward(ids, dy, V, scale, first, dtype, base.nan_to_num(0))
    ref.check(got[~absent], want[~absent], tol[~absent], "added")


@pytest.mark.parametrize("T", [64, 1000, 2048, 5000])
def test_all_tokens_of_one_row_and_of_none(jet, T):
    g = _gen(T)
    dy = _normal(g, (T, 1032))
    for ids in (torch.full((T,), 3, device="cuda"), torch.full((T,), 0, device="cuda"), torch.full((T,), -1, device="cuda"),
                torch.full((T,), 2 ** 62, device="cuda"), torch.arange(T, device="cuda") % 2 * 3):
        dw = jet.embedding_bwd(ids, dy, 4)
        ref.check(dw, *ref.embedding_backward(ids, dy, 4, 1.0, 0, f32), "dw")
        assert _same(dw, jet.embedding_bwd(ids, dy, 4))                  # no atomic sums


def test_rows_of_one_token_are_exact(jet):
    """Distinct ids in random order: every row of the gradient is one of dy's, whichever path sorts them."""
    for T in (50, 1000, 4097, 20000):
        g = _gen(T)
        ids, dy = torch.randperm(T, generator=g, device="cuda"), _normal(g, (T, 72))
        for dtype in (bf, f32):
            dw = jet.embedding_bwd(ids, dy, T, dtype=dtype)
            assert torch.equal(dw[ids], dy.to(dtype))


def test_a_table_past_32_bits(jet):
    """Rows that lie more than 2^32 bytes into the table, and zeros there."""
    V, H = 70001, 16384
    ids = torch.tensor([70000, 0, 69999, 70000], device="cuda")
    dy = _normal(_gen(1), (4, H))
    dw = jet.embedding_bwd(ids, dy, V)
    assert torch.equal(dw[69999], dy[2].float()) and torch.equal(dw[70000], dy[0].float() + dy[3].float()) and torch.equal(dw[0], dy[1].float())
    assert int((dw != 0).any(dim=1).sum()) == 3
    assert torch.equal(jet.embedding_fwd(ids, dw), dw[ids].to(bf))


# ---------------------------------------------------------------------- norms

NORMS = [(1, 4096), (1, 8), (3, 72), (5, 128), (37, 512), (513, 512), (700, 520), (9, 1000), (600, 1024), (1001, 1032), (513, 2048), (4, 2056), (515, 4096), (600, 4104),
         (1500, 5120), (2, 8192), (513, 8192), (514, 8200), (3, 16384), (520, 16392), (5, 32768), (530, 32768)]
EPS = 1e-5


def _rows(gen, M, K):
    """Hidden states: a mean, channels far larger than the others; a row of zeros, one of equal values, one of large ones."""
    x = torch.randn((M, K), generator=gen, device="cuda") + 0.3
    x[:, ::97] *= 50
    if M > 4:
        x[1] = 0
        x[2] = 1000.0
        x[3] *= 1e18
        x[4] += 300
    return x.to(bf)


@pytest.mark.parametrize("M,K", NORMS)
def test_layernorm_fwd(jet, M, K):
    g = _gen(M + K)
    x, gamma, beta, res = _rows(g, M, K), 1 + _normal(g, (K,), 0.2), _normal(g, (K,), 0.1), _normal(g, (M, K))
    for b, r in ((beta, None), (None, None), (beta, res)):
        o = jet.layernorm_fwd(x, gamma, b, EPS, r)
        assert set(o) == ({"y"} if r is None else {"y", "sum"})
        s = x
        if r is not None:
            s = (x.double() + r.double()).to(f32).to(bf)                 # binary32 holds the sum of two bf16 numbers or rounds it
            off = (o["sum"].double() - (x.double() + r.double())).abs()
            assert (off <= (x.double() + r.double()).abs() * (ref.BF + ref.F)).all()
            s = o["sum"]
        ref.check(o["y"], *ref.layer_norm(s, gamma, b, EPS), "y")
        if K % 128 == 0:
            q = jet.layernorm_fwd(x, gamma, b, EPS, r, quant=True)
            assert set(q) == ({"q_row", "s_row"} if r is None else {"q_row", "s_row", "sum"})
            want = jet.quant_act(o["y"])
            assert _same(q["q_row"], want["q_row"]) and _same(q["s_row"], want["s_row"])
            assert r is None or _same(q["sum"], o["sum"])


@pytest.mark.parametrize("M,K", NORMS)
@pytest.mark.parametrize("layer", [True, False])
def test_norm_bwd(jet, M, K, layer):
    g = _gen(M + K + 1)
    x, gamma, dy, dres = _rows(g, M, K), 1 + _normal(g, (K,), 0.2), _normal(g, (M, K), 1e-3), _normal(g, (M, K), 1e-3)
    f = jet.layernorm_bwd if layer else jet.rmsnorm_bwd
    for r in (None, dres):
        got = f(dy, x, gamma, EPS, r)
        want, tol = ref.norm_backward(dy, x, gamma, EPS, r, layer)
        assert len(got) == (3 if layer else 2)
        for a, b, t, name in zip(got, want, tol, ("dx", "dgamma", "dbeta")):
            ref.check(a, b, t, name)
        assert all(_same(a, b) for a, b in zip(got, f(dy, x, gamma, EPS, r)))


def test_norm_gradients_against_differences(jet):
    """dx, dgamma and dbeta of a loss, against central differences of the formulas in 64 bits."""
    g = _gen(5)
    M, K = 3, 16
    x, gamma, beta, dy = _normal(g, (M, K)), 1 + _normal(g, (K,), 0.2), _normal(g, (K,), 0.2), _normal(g, (M, K))

    def loss(x, gamma, beta, layer):
        c = x - x.mean(dim=1, keepdim=True) if layer else x
        return ((c / torch.sqrt((c * c).mean(dim=1, keepdim=True) + EPS) * gamma + beta) * dy.double()).sum()

    h = 1e-6
    for layer, grads in ((True, jet.layernorm_bwd(dy, x, gamma, EPS)), (False, jet.rmsnorm_bwd(dy, x, gamma, EPS))):
        at = [x.double(), gamma.double(), beta.double()]
        for k, grad in enumerate(grads):
            num = torch.zeros(at[k].numel(), dtype=f64, device="cuda")
            for i in range(num.numel()):
                e = torch.zeros_like(num)
                e[i] = h
                up, down = list(at), list(at)
                up[k], down[k] = at[k] + e.view_as(at[k]), at[k] - e.view_as(at[k])
                num[i] = (loss(*up, layer) - loss(*down, layer)) / (2 * h)
            # differences: h^2 of a third derivative, and 2^-52 of the loss over h; the result's own rounding
            off = 1e-6 + grad.double().abs().flatten() * (ref.BF if k == 0 else 8 * ref.F) * 1.01
            assert ((grad.double().flatten() - num).abs() <= off).all(), (layer, k)


@pytest.mark.parametrize("K", [512, 2048, 4096])
def test_a_row_gets_the_same_bytes_among_others(jet, K):
    """Few rows and many take other kernels; those of one kernel give a row the same bytes wherever it is."""
    g = _gen(K)
    x, gamma, beta, dy = _rows(g, 700, K), 1 + _normal(g, (K,), 0.2), _normal(g, (K,), 0.1), _normal(g, (700, K))
    y = jet.layernorm_fwd(x, gamma, beta, EPS)["y"]
    assert _same(jet.layernorm_fwd(x[:600].contiguous(), gamma, beta, EPS)["y"], y[:600])
    dx = jet.layernorm_bwd(dy, x, gamma, EPS)[0]
    assert _same(jet.layernorm_bwd(dy[7:8].contiguous(), x[7:8].contiguous(), gamma, EPS)[0], dx[7:8])


# ---------------------------------------------------------- norm and clipping

def _grads(gen, sizes, std=1e-3):
    return [_normal(gen, n if isinstance(n, tuple) else (n,), std, bf if i % 3 else f32) for i, n in enumerate(sizes)]


# elements of the tensors; the first, fourth, ... are f32: single elements and none, ends of a chunk, more tensors than one launch has
CLIP = [[1], [3, 5, 7], [0, 17, 0], [8192, 8192, 8192], [8191, 8193, 16385, 4096], [(300, 1000), (1000, 4096), 1, 100000], [7 * i % 50 for i in range(145)],
        [(i * 37) % 20000 + 1 for i in range(500)], [20_000_000, 30_000_001]]


@pytest.mark.parametrize("sizes", CLIP, ids=lambda s: str(len(s)) + "x" + str(s[0]))
def test_norm_and_clipping(jet, sizes):
    g = _gen(len(sizes))
    grads = _grads(g, sizes)
    want = ref.norm(grads)
    norm = jet.grad_norm(grads)
    assert norm.shape == () and norm.dtype == f32 and abs(norm.item() - want) <= want * ref.F * 1.01
    for max_norm in (0.3 * want, 3.0 * want, 0.0, math.inf):
        to = [torch.full_like(t, 9.0) for t in grads]
        assert _same(jet.clip_grads(grads, max_norm, out=to), norm)
        max32 = _f32(max_norm)
        for a, b, t in zip(to, *ref.clipped(grads, max32)):
            ref.check(a, b, t, "out")
        mine = [t.clone() for t in grads]
        assert _same(jet.clip_grads(tuple(mine), max_norm), norm)        # in place
        assert all(_same(a, b) for a, b in zip(mine, to))
        if max_norm > want:
            assert all(_same(a, b) for a, b in zip(to, grads))
        given = torch.tensor([2 * _f32(want)], device="cuda")            # the norm of all shards
        mine = [t.clone() for t in grads]
        assert jet.clip_grads(mine, max_norm, norm=given) is given
        for a, b, t in zip(mine, *ref.clipped(grads, max32, given.item())):
            ref.check(a, b, t, "given")


@pytest.mark.parametrize("value", [math.inf, -math.inf, math.nan])
def test_a_norm_that_is_not_finite_leaves_the_values(jet, value):
    grads = _grads(_gen(3), [1000, 9000, 5])
    grads[1][8999] = value
    before = [t.clone() for t in grads]
    norm = jet.clip_grads(grads, 1e-9)
    assert not math.isfinite(norm.item()) and math.isnan(norm.item()) == math.isnan(value)
    assert all(_same(a, b) for a, b in zip(grads, before))
    to = [torch.zeros_like(t) for t in grads]
    jet.clip_grads(grads, 1e-9, out=to)
    assert all(_same(a, b) for a, b in zip(to, before))
    for bad in (math.inf, math.nan):
        jet.clip_grads(grads, 1.0, norm=torch.tensor(bad, device="cuda"))
        assert all(_same(a, b) for a, b in zip(grads, before))


def test_squares_outside_binary32(jet):
    for v in (1e30, 1e-30):
        grads = [torch.full((5000,), v, dtype=t, device="cuda") for t in (bf, f32)]
        want = ref.norm(grads)
        assert abs(jet.grad_norm(grads).item() - want) <= want * ref.F * 1.01
        assert abs(jet.clip_grads(grads, 0.5 * want).item() - want) <= want * ref.F * 1.01
        assert abs(ref.norm(grads) - 0.5 * want) <= 0.5 * want * (ref.BF + 4 * ref.F)
    big = [torch.full((4,), 3e38, device="cuda")]                        # the norm itself is beyond binary32
    before = big[0].clone()
    assert math.isinf(jet.clip_grads(big, 1.0).item()) and _same(big[0], before)
