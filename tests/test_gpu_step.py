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
EMBED = [(1, 4096, 500, 0), (1, 8, 1, 0), (2, 72, 3, 0), (37, 64, 50, 7), (64, 136, 20, 0), (65, 136, 20, 0), (100, 1000, 9, -3), (256, 520, 30, 0), (257, 520, 30, 2),
         (1000, 520, 7001, 0), (1023, 8, 300, 0), (1024, 128, 5000, 0), (1025, 128, 60, 100), (3001, 264, 40, 0), (5000, 2056, 1234, 11), (9000, 24, 100000, 0),
         (33000, 40, 7, 0), (9000, 8, 5000001, -(1 << 40)), (20001, 4104, 3000, 0), (16400, 1544, 900, 0),
         (65537, 72, 4000, 0), (530000, 16, 70000, -9), (1000, 2568, 3, 0), (700, 4104, 9000, 0), (1024, 2048, 2, 0)]
ONE_ROW = [64, 256, 1000, 2048, 5000, 70000, 524289]
PAST_THE_CACHES = [(16385, 4096)]


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


@pytest.mark.parametrize("T", ONE_ROW)
def test_all_tokens_of_one_row_and_of_none(jet, T):
    g = _gen(T)
    dy = _normal(g, (T, 1032 if T < 10000 else 40))
    for ids in (torch.full((T,), 3, device="cuda"), torch.full((T,), 0, device="cuda"), torch.full((T,), -1, device="cuda"),
                torch.full((T,), 2 ** 62, device="cuda"), torch.arange(T, device="cuda") % 2 * 3):
        dw = jet.embedding_bwd(ids, dy, 4)
        ref.check(dw, *ref.embedding_backward(ids, dy, 4, 1.0, 0, f32), "dw")
        assert _same(dw, jet.embedding_bwd(ids, dy, 4))                  # no atomic sums


def test_rows_of_one_token_are_exact(jet):
    """Distinct ids in random order: every row of the gradient is one of dy's, whichever path sorts them."""
    for T in (50, 320, 1000, 4097, 20000, 100001, 1000001):
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
         (1500, 5120), (2, 8192), (513, 8192), (514, 8200), (3, 16384), (520, 16392), (5, 32768), (530, 32768), (20001, 64), (1025, 1024), (5000, 2560),
         (9, 4096), (700, 12288), (1500, 2048), (2100, 8192), (1100, 4104)]
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


@pytest.mark.parametrize("M,K", PAST_THE_CACHES)
def test_outputs_that_are_written_past_the_caches(jet, M, K):
    g = _gen(M)
    x, gamma, beta, dy = _rows(g, M, K), 1 + _normal(g, (K,), 0.2), _normal(g, (K,), 0.1), _normal(g, (M, K), 1e-3)
    ref.check(jet.layernorm_fwd(x, gamma, beta, EPS)["y"], *ref.layer_norm(x, gamma, beta, EPS), "y")
    for f, layer in ((jet.layernorm_bwd, True), (jet.rmsnorm_bwd, False)):
        got = f(dy, x, gamma, EPS)
        for a, b, t, name in zip(got, *ref.norm_backward(dy, x, gamma, EPS, None, layer), ("dx", "dgamma", "dbeta")):
            if b is not None:
                ref.check(a, b, t, name)
        assert _same(f(dy[:300].contiguous(), x[:300].contiguous(), gamma, EPS)[0], got[0][:300])
    ids = torch.randint(-5, 1005, (M,), generator=g, device="cuda")
    for dtype in (bf, f32):
        w = _normal(g, (1000, K), 0.02, dtype)
        ref.check(jet.embedding_fwd(ids, w, 3.0), *ref.embedding(ids, w, 3.0, 0), "embedding")


def test_values_that_are_not_finite_stay_in_their_rows(jet):
    g = _gen(9)
    for M, K in ((9, 512), (9, 1024), (9, 2056), (900, 1024)):
        x, gamma, beta, dy = _normal(g, (M, K)), 1 + _normal(g, (K,), 0.2), _normal(g, (K,)), _normal(g, (M, K))
        bad = x.clone()
        bad[4, K // 2], bad[5, 3], bad[6] = math.nan, math.inf, -math.inf
        rest = torch.ones(M, dtype=torch.bool, device="cuda")
        rest[4:7] = False
        y = jet.layernorm_fwd(bad, gamma, beta, EPS)["y"]
        assert _same(y[rest], jet.layernorm_fwd(x, gamma, beta, EPS)["y"][rest]) and y[~rest].isnan().all()
        if K % 128 == 0:
            q, want = jet.layernorm_fwd(bad, gamma, beta, EPS, quant=True), jet.quant_act(y)
            assert _same(q["q_row"], want["q_row"]) and _same(q["s_row"], want["s_row"])
        for f in (jet.layernorm_bwd, jet.rmsnorm_bwd):
            got = f(dy, bad, gamma, EPS)[0]
            assert _same(got[rest], f(dy, x, gamma, EPS)[0][rest]) and got[~rest].isnan().any(dim=1).all()
    for T in (200, 700, 3000):
        ids = torch.arange(T, device="cuda") % 50
        ids[::7] = -1
        dy = _normal(g, (T, 264))
        dirty = dy.clone()
        dirty[::7] = math.nan                                            # padding
        clean = jet.embedding_bwd(ids, dy, 50)
        assert _same(jet.embedding_bwd(ids, dirty, 50), clean)
        t = int((ids == 20).nonzero()[0])
        dirty[t, 5] = math.inf
        got = jet.embedding_bwd(ids, dirty, 50)
        others = torch.arange(50, device="cuda") != 20
        assert _same(got[others], clean[others]) and got[20, 5].isinf() and got[20].isfinite().sum() == 263


def test_subnormal_values(jet):
    g = _gen(4)
    w = _normal(g, (50, 64), 1e-39, f32)
    ids = torch.arange(50, device="cuda")
    ref.check(jet.embedding_fwd(ids, w), *ref.embedding(ids, w, 1.0, 0), "y")
    dy = _normal(g, (50, 64), 1e-39)
    for dtype in (bf, f32):
        ref.check(jet.embedding_bwd(ids % 7, dy, 7, dtype=dtype), *ref.embedding_backward(ids % 7, dy, 7, 1.0, 0, dtype), "dw")
    grads = [_normal(g, (100,), 1e-39, t) for t in (bf, f32)]
    want = ref.norm(grads)
    to = [torch.empty_like(t) for t in grads]
    norm = jet.clip_grads(grads, 0.5 * want, out=to)
    assert abs(norm.item() - want) <= want * ref.F * 1.01 + ref.LEAST[f32]
    for a, b, t in zip(to, *ref.clipped(grads, _f32(0.5 * want))):
        ref.check(a, b, t, "out")


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


SAME_BYTES, MANY = [64, 512, 520, 1000, 1024, 1032, 2048, 2560, 4096, 4608, 5120, 7000, 8192, 16384, 20000], 1100


@pytest.mark.parametrize("K", SAME_BYTES)
def test_a_row_gets_the_same_bytes_in_every_call(jet, K):
    """Rollout and training: alone and among many, which take other kernels."""
    g = _gen(K)
    M = MANY
    x, gamma, beta, dy, res = _rows(g, M, K), 1 + _normal(g, (K,), 0.2), _normal(g, (K,), 0.1), _normal(g, (M, K)), _normal(g, (M, K))
    for r in (None, res):
        many = jet.layernorm_fwd(x, gamma, beta, EPS, r)
        for a, b in ((0, 1), (5, 42), (M - 700, M)):
            few = jet.layernorm_fwd(x[a:b].contiguous(), gamma, beta, EPS, None if r is None else r[a:b].contiguous())
            assert all(_same(few[k], many[k][a:b]) for k in many)
    for f in (jet.layernorm_bwd, jet.rmsnorm_bwd):
        dx = f(dy, x, gamma, EPS)[0]
        for a, b in ((7, 8), (0, 600)):
            assert _same(f(dy[a:b].contiguous(), x[a:b].contiguous(), gamma, EPS)[0], dx[a:b])


# ---------------------------------------------------------- norm and clipping

def _grads(gen, sizes, std=1e-3):
    return [_normal(gen, n if isinstance(n, tuple) else (n,), std, bf if i % 3 else f32) for i, n in enumerate(sizes)]


# elements of the tensors; the first, fourth, ... are f32: single elements and none, ends of a chunk, more tensors than one launch has
CLIP = [[1], [3, 5, 7], [0, 17, 0], [8192, 8192, 8192], [8191, 8193, 16385, 4096], [(300, 1000), (1000, 4096), 1, 100000], [7 * i % 50 for i in range(145)],
        [(i * 37) % 20000 + 1 for i in range(500)], [20_000_000, 30_000_001],
        [50_000_000, 70_000_001], [1_000_000 + i for i in range(150)]]


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


def test_tensors_past_32_bits(jet):
    """Activations and gradients of more than 2^32 bytes: the last rows are what they are alone."""
    g = _gen(6)
    M, K = 530_000, 4104
    x, res = torch.empty((M, K), dtype=bf, device="cuda"), torch.zeros((M, K), dtype=bf, device="cuda")
    x.copy_(_normal(g, (1, K)).expand(M, K))
    x[-5:], res[-5:] = _normal(g, (5, K)), _normal(g, (5, K))
    gamma, beta, last = 1 + _normal(g, (K,), 0.2), _normal(g, (K,), 0.1), slice(M - 5, M)
    o, few = jet.layernorm_fwd(x, gamma, beta, EPS, res), jet.layernorm_fwd(x[last].contiguous(), gamma, beta, EPS, res[last].contiguous())
    assert all(_same(o[k][last], few[k]) for k in few)
    assert _same(jet.layernorm_fwd(x, gamma, beta, EPS)["y"][last], jet.layernorm_fwd(x[last].contiguous(), gamma, beta, EPS)["y"])
    del o
    for f in (jet.layernorm_bwd, jet.rmsnorm_bwd):                       # res as dy: zeros but for the last rows, whose normalized values are below 6
        got, few = f(res, x, gamma, EPS, x), f(res[last].contiguous(), x[last].contiguous(), gamma, EPS, x[last].contiguous())
        assert _same(got[0][last], few[0])
        for a, b in zip(got[1:], few[1:]):
            assert torch.allclose(a, b, rtol=0, atol=20 * ref.F * float(res[last].double().abs().sum(dim=0).max()) * 6)
    del got, few
    ids = torch.full((M,), -1, device="cuda")
    ids[-5:] = torch.tensor([4, 0, 3, 1, 2], device="cuda")
    dw = jet.embedding_bwd(ids, res, 5)
    assert torch.equal(dw[ids[-5:]], res[last].float())
    assert torch.equal(jet.embedding_fwd(ids, dw)[last], res[last])
    del x, dw
    n = (1 << 31) + 9
    big = res.view(-1)[:1].expand(n).contiguous()
    big.fill_(1.0)
    assert abs(jet.grad_norm([big]).item() - math.sqrt(n)) <= math.sqrt(n) * ref.F * 1.01
    jet.clip_grads([big], 0.5 * math.sqrt(n))
    assert bool((big == 0.5).all())


# ------------------------------------------------------------------- together

def _step(jet, w, ids, dh):
    """A training step of two pre-norm blocks: what stands in front of them, between them and behind them, with FP8 MLPs as the blocks and
    one norm of each kind.  Returns the final state and the clipped gradients."""
    from paper_2601_14243_amd import mlp_block
    mlp = w["mlp"]
    x0 = jet.embedding_fwd(ids, w["table"], w["scale"])
    n0 = jet.layernorm_fwd(x0, w["gamma"][0], w["beta"][0], EPS)["y"]
    y0, s0 = mlp_block.forward(n0, mlp[0])
    r1 = jet.layernorm_fwd(y0, w["gamma"][1], w["beta"][1], EPS, residual=x0)
    y1, s1 = mlp_block.forward(r1["y"], mlp[1])
    last = jet.layernorm_fwd(y1, w["gamma"][2], None, EPS, residual=r1["sum"])
    d2, dg2, db2 = jet.layernorm_bwd(dh, last["sum"], w["gamma"][2], EPS)
    g1 = mlp_block.backward(s1, d2, mlp[1])
    d1, dg1, db1 = jet.layernorm_bwd(g1["dx"], r1["sum"], w["gamma"][1], EPS, dres=d2)
    g0 = mlp_block.backward(s0, d1, mlp[0])
    d0, dg0, db0 = jet.layernorm_bwd(g0["dx"], x0, w["gamma"][0], EPS, dres=d1)
    dw = jet.embedding_bwd(ids, d0, w["table"].shape[0], w["scale"])
    grads = [dw, g0["dw_gu"], g0["dw_d"], g1["dw_gu"], g1["dw_d"], dg0, db0, dg1, db1, dg2, db2]
    to = [torch.empty_like(t) for t in grads]
    norm = jet.clip_grads(grads, w["max_norm"], out=to)
    kept = dict(x0=x0, n0=n0, y0=y0, r1=r1, y1=y1, last=last, d2=d2, g1=g1, d1=d1, g0=g0, d0=d0, dw=dw, dgamma=(dg0, dg1, dg2), dbeta=(db0, db1, db2), grads=grads)
    return [last["y"], norm, *to], kept


def _step_inputs(seed, T=256, H=256, I=512, V=300):
    from paper_2601_14243_amd import mlp_block
    g = _gen(seed)
    w = dict(table=_normal(g, (V, H), 0.05, f32), scale=_f32(math.sqrt(H)), gamma=[1 + _normal(g, (H,), 0.1) for _ in range(3)],
             beta=[_normal(g, (H,), 0.1) for _ in range(2)], max_norm=1e-3,
             mlp=[mlp_block.MlpWeights(_normal(g, (2 * I, H), 0.05), _normal(g, (H, I), 0.05)) for _ in range(2)])
    return w, torch.randint(0, V, (T,), generator=g, device="cuda"), _normal(g, (T, H), 1e-2)


def test_a_training_step(jet):
    w, ids, dh = _step_inputs(11)
    out, k = _step(jet, w, ids, dh)
    V = w["table"].shape[0]
    ref.check(k["x0"], *ref.embedding(ids, w["table"], w["scale"], 0), "x0")
    for y, x, i in ((k["n0"], k["x0"], 0), (k["r1"]["y"], k["r1"]["sum"], 1), (k["last"]["y"], k["last"]["sum"], 2)):
        ref.check(y, *ref.layer_norm(x, w["gamma"][i], w["beta"][i] if i < 2 else None, EPS), f"norm {i}")
    assert torch.equal(k["r1"]["sum"], k["y0"] + k["x0"]) and torch.equal(k["last"]["sum"], k["y1"] + k["r1"]["sum"])
    for i, (dx, dy, x, dres) in enumerate(((k["d0"], k["g0"]["dx"], k["x0"], k["d1"]), (k["d1"], k["g1"]["dx"], k["r1"]["sum"], k["d2"]),
                                           (k["d2"], dh, k["last"]["sum"], None))):
        want, tol = ref.norm_backward(dy, x, w["gamma"][i], EPS, dres, True)
        for a, b, t, name in zip((dx, k["dgamma"][i], k["dbeta"][i]), want, tol, ("dx", "dgamma", "dbeta")):
            ref.check(a, b, t, f"{name} {i}")
    ref.check(k["dw"], *ref.embedding_backward(ids, k["d0"], V, w["scale"], 0, f32), "dw")
    assert abs(out[1].item() - ref.norm(k["grads"])) <= ref.norm(k["grads"]) * ref.F * 1.01 and out[1].item() > w["max_norm"]
    for a, b, t in zip(out[2:], *ref.clipped(k["grads"], _f32(w["max_norm"]))):
        ref.check(a, b, t, "clipped")


def test_a_training_step_replayed_from_two_graphs(jet):
    """Both graphs' pools hold their scratch memory; replays in turn, with eager work in between, give what the eager step gives."""
    w, ids, dh = _step_inputs(12)
    inputs = [_step_inputs(20 + i)[1:] for i in range(3)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        _step(jet, w, ids, dh)
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graphs = []
    pool = torch.cuda.graph_pool_handle()
    for _ in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, pool=pool):
            out, _ = _step(jet, w, ids, dh)
        graphs.append((g, out))
    for rep in range(6):
        a, b = inputs[rep % 3]
        ids.copy_(a)
        dh.copy_(b)
        g, out = graphs[rep % 2]
        g.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in out]
        want, _ = _step(jet, w, ids, dh)
        torch.cuda.synchronize()
        assert all(_same(p, q) for p, q in zip(got, want)), rep


def test_every_way_of_a_call_replayed_from_a_graph(jet):
    """Few, more, many and very many tokens; several launches of clipping; rows of every team; other inputs in each replay."""
    g = _gen(50)
    tokens = [(200, 264), (900, 520), (1000, 4104), (9000, 1032), (70000, 72)]
    ids, dy = [torch.zeros(T, dtype=i64, device="cuda") for T, _ in tokens], [_normal(g, t) for t in tokens]
    rows = [(300, 512), (700, 1024), (1030, 4096), (3, 16384), (2, 32768)]
    x, gamma = [_normal(g, r) for r in rows], [1 + _normal(g, (r[1],), 0.2) for r in rows]
    grads = _grads(g, [1000 + i for i in range(300)])

    def calls():
        out = [jet.embedding_bwd(i, d, 3000, 0.5, 7) for i, d in zip(ids, dy)]
        for v, w in zip(x, gamma):
            out += [*jet.layernorm_fwd(v, w, None, EPS, v).values(), *jet.layernorm_bwd(v, v, w, EPS), *jet.rmsnorm_bwd(v, v, w, EPS, v)]
        to = [torch.empty_like(t) for t in grads]
        return [*out, jet.clip_grads(grads, 1e-3, out=to), jet.grad_norm(grads), *to]

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        calls()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = calls()
    for rep in range(4):
        for i in ids:
            i.copy_(torch.randint(0, 40 if rep % 2 else 3100, i.shape, generator=g, device="cuda"))
        for t in (*dy, *x, *grads):
            t.copy_(_normal(g, t.shape, 1.0, t.dtype))
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in out]
        assert all(_same(a, b) for a, b in zip(got, calls())), rep


def test_calls_on_a_stream_of_the_callers(jet):
    """Work of another stream that is waited for, two streams at once, and scratch memory of a call that the next one gets."""
    want = {}
    cases = [_step_inputs(30 + i) for i in range(2)]
    for i, c in enumerate(cases):
        want[i] = [t.clone() for t in _step(jet, *c)[0]]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = {}
    for rep in range(3):
        for i, s in enumerate(streams):
            s.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(s):
                got[i] = _step(jet, *cases[i])[0]
        for s in streams:
            torch.cuda.current_stream().wait_stream(s)
        torch.cuda.synchronize()
        for i in got:
            assert all(_same(a, b) for a, b in zip(got[i], want[i])), (rep, i)


def test_unaligned_and_overlapping_tensors_are_refused(jet):
    x = torch.zeros(4 * 64 + 8, dtype=bf, device="cuda")
    off, gamma, ids = x[1:257].view(4, 64), torch.ones(64, dtype=bf, device="cuda"), torch.zeros(4, dtype=i64, device="cuda")
    for call in (lambda: jet.embedding_fwd(ids, off), lambda: jet.embedding_bwd(ids, off, 9), lambda: jet.layernorm_fwd(off, gamma, None, EPS),
                 lambda: jet.layernorm_bwd(off, off, gamma, EPS), lambda: jet.rmsnorm_bwd(x[:256].view(4, 64), off, gamma, EPS), lambda: jet.grad_norm([gamma, off]),
                 lambda: jet.clip_grads([off], 1.0)):
        with pytest.raises(jet.JetError, match="status 3"):
            call()
    for grads, out in (([gamma, gamma], None), ([x[:64], x[32:96]], None), ([gamma], [gamma])):
        with pytest.raises(jet.JetError, match="status 4"):
            jet.clip_grads(grads, 1.0, out=out)
    assert abs(jet.grad_norm([gamma, gamma]).item() - math.sqrt(128)) < 1e-5             # only read: counted twice
    for call in (lambda: jet.embedding_fwd(ids[:0], gamma.view(1, 64)), lambda: jet.layernorm_fwd(x[:0].view(0, 64), gamma, None, EPS),
                 lambda: jet.layernorm_fwd(x[:120].view(2, 60), gamma[:60], None, EPS), lambda: jet.layernorm_fwd(x[:256].view(4, 64), gamma, None, EPS, quant=True)):
        with pytest.raises(jet.JetError, match="status [12]"):           # torch gives an empty tensor no address
            call()


@pytest.mark.parametrize("native", [True, False])
def test_same_results_from_the_native_and_the_python_path(jet, monkeypatch, native):
    from paper_2601_14243_amd import binding
    g = _gen(40)
    x, gamma, dy, ids = _normal(g, (300, 256)), 1 + _normal(g, (256,), 0.2), _normal(g, (300, 256)), torch.randint(-2, 60, (300,), generator=g, device="cuda")
    w, grads = _normal(g, (50, 256), 1.0, f32), _grads(g, [1000, 5, 0, 300])
    two = torch.tensor(2.0, device="cuda")

    def calls():
        yield jet.embedding_fwd(ids, w, 2.0, 3)
        yield jet.embedding_fwd(ids.int(), w.to(bf), 2, first=0, out=torch.zeros((300, 256), dtype=bf, device="cuda"))
        yield jet.embedding_bwd(ids, dy, 50, 0.5)
        yield jet.embedding_bwd(ids, dy, 50, 1, 4, bf, out=w.to(bf), accumulate=True)
        for quant in (False, True):
            for res in (None, dy):
                yield jet.layernorm_fwd(x, gamma, None if quant else gamma, 1e-5, res, quant)
        yield jet.layernorm_bwd(dy, x, gamma, 1e-5, dy)
        yield jet.rmsnorm_bwd(dy, x, gamma, 1)
        yield jet.grad_norm(grads)
        for kw in (dict(), dict(out=tuple(torch.zeros_like(t) for t in grads)), dict(norm=two)):
            mine = [t.clone() for t in grads]
            r = jet.clip_grads(mine, 1e-3, **kw)
            assert kw.get("norm") is None or r is two
            yield (r, *mine, *kw.get("out", ()))

    flat = lambda r: [r[k] for k in sorted(r)] if isinstance(r, dict) else list(r) if isinstance(r, tuple) else [r]
    want = [[t.clone() for t in flat(r)] for r in calls()]
    if not native:
        monkeypatch.setattr(binding, "_host", type("Declines", (), {"__getattr__": lambda self, name: lambda *a: None})())
    for i, (r, q) in enumerate(zip(calls(), want)):
        r = flat(r)
        assert len(r) == len(q) and all(_same(a, c) and a.device == c.device for a, c in zip(r, q)), i
