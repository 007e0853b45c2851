"""Long sums of the operators of a training step, on values whose sums binary32 holds: whatever the order, a term that is lost, doubled or
put to another row or column shows, where a bound on the roundings of so many terms would let it pass."""
import pytest
import torch

import step_ref as ref
import test_gpu_step as gpu
from test_gpu_step import _gen, _ids, _normal, _same, bf, f32, f64, i32, i64, jet  # noqa: F401

pytestmark = pytest.mark.gpu
SMALL = 3                                                                # magnitude of the terms: a sum of up to 2^22 stays below 2^24


def _whole(gen, shape):
    """Whole numbers of -SMALL .. SMALL without zero, as bf16."""
    v = torch.randint(1, 2 * SMALL + 1, shape, generator=gen, device="cuda")
    return torch.where(v > SMALL, SMALL - v, v).to(bf)


def _embedding_sum(ids, dy, rows, first):
    """Sums for each row of the table, in 64 bits."""
    row, here = ref.in_shard(ids, first, rows)
    d = dy.to(f64).masked_fill(~here[:, None], 0)
    return torch.zeros((rows, dy.shape[1]), dtype=f64).index_add(0, row.cpu(), d.cpu()).to("cuda")


def _check_embedding(jet, gen, ids, T, H, V, first):
    dy, scale = _whole(gen, (T, H)), 0.25
    want = _embedding_sum(ids, dy, V, first) * scale
    assert float(want.abs().max()) * 4 < 1 << 24
    base = torch.randint(-99, 100, (V, H), generator=gen, device="cuda") * scale
    for dtype in (f32, bf):
        assert _same(jet.embedding_bwd(ids, dy, V, scale, first, dtype) + 0, want.to(f32).to(dtype) + 0)        # (+ 0: no sign of a zero)
        got = jet.embedding_bwd(ids, dy, V, scale, first, out=base.to(dtype, copy=True), accumulate=True)
        assert _same(got + 0, (base + want).to(f32).to(dtype) + 0)


@pytest.mark.parametrize("T,H,V,first", gpu.EMBED)
def test_embedding_bwd_of_whole_numbers(jet, T, H, V, first):
    g = _gen(T + H)
    wide = T % 2 or abs(first) > 1 << 30                                 # ids that 32 bits hold
    _check_embedding(jet, g, _ids(g, T, V, first, i64 if wide else i32), T, H, V, first)


@pytest.mark.parametrize("T,H", [(64, 1032), (256, 1032), (257, 1032), (1000, 1032), (1000, 4104), (1025, 1032), (2048, 1032), (5000, 1032), (16400, 2056), (40000, 4104),
                                 (70000, 520), (140000, 264), (524289, 40), (1100000, 8)])
def test_embedding_bwd_of_frequent_ids(jet, T, H):
    """Rows that nearly all tokens have, as of padding: all on one, in turn on two, long runs with others in between."""
    g = _gen(T)
    at = torch.arange(T, device="cuda")
    often = torch.where(torch.rand((T,), generator=g, device="cuda") < 0.01, torch.randint(0, 60, (T,), generator=g, device="cuda"), 33)
    for ids in (torch.full((T,), 3, device="cuda"), at % 2 * 3, often, at * 7 // T):
        _check_embedding(jet, g, ids, T, H, 64, 0)


def _signs(gen, M, K):
    """Rows of as many 1 as -1, times a power of two for each row: mean 0, and 1 / rms is that power's inverse."""
    s = torch.randint(0, 2, (M, K // 2), generator=gen, device="cuda") * 2 - 1
    s = torch.cat((s, -s), dim=1)[:, torch.randperm(K, generator=gen, device="cuda")]
    return s, (s * torch.exp2(torch.randint(-8, 9, (M, 1), generator=gen, device="cuda").to(f32))).to(bf)


@pytest.mark.parametrize("M,K", [(1, 64), (5, 512), (20001, 64), (3000, 512), (1001, 1024), (9000, 1024), (1001, 2048), (4096, 4096), (2100, 8192), (530, 16384),
                                 (2000, 16384), (530, 32768), (1100, 32768)])
def test_norm_sums_of_whole_numbers(jet, M, K):
    """With columns in a power of two all steps up to n = 1 or -1 are exact, and so are both gradients."""
    g = _gen(M + K)
    n, x = _signs(g, M, K)
    dy, gamma, dres = _whole(g, (M, K)), 1 + _normal(g, (K,), 0.2), _normal(g, (M, K))
    dgamma, dbeta = (dy.to(f64) * n).sum(dim=0).to(f32), dy.to(f64).sum(dim=0).to(f32)
    for r in (None, dres):
        got = jet.layernorm_bwd(dy, x, gamma, 0.0, r)
        assert torch.equal(got[1], dgamma) and torch.equal(got[2], dbeta)
        assert torch.equal(jet.rmsnorm_bwd(dy, x, gamma, 0.0, r)[1], dgamma)


@pytest.mark.parametrize("M,K", gpu.NORMS)
def test_norm_sums_lose_no_row(jet, M, K):
    """Any number of columns: dbeta is exact, dgamma a whole number but for roundings that are less than half."""
    g = _gen(M + K + 2)
    n, x = _signs(g, M, K)
    dy, gamma = _whole(g, (M, K)), 1 + _normal(g, (K,), 0.2)
    dgamma, dbeta = (dy.to(f64) * n).sum(dim=0), dy.to(f64).sum(dim=0)
    # n as in step_ref, with an exact mean; the additions of a workgroup, which takes 40 rows at most, of sums of at most SMALL for each; the last rounding
    assert M <= 40 * 512
    off_n = 2 * ref.F + (ref.ADD + 2 * ref.F) / 2 + 2 * ref.F
    off = off_n * dy.to(f64).abs().sum(dim=0) + M * ref.F * SMALL * 40 * 1.01 + ref.F * dgamma.abs()
    assert float(off.max()) < 0.5
    got = jet.layernorm_bwd(dy, x, gamma, 0.0)
    assert torch.equal(got[2], dbeta.to(f32))
    for a in (got[1], jet.rmsnorm_bwd(dy, x, gamma, 0.0)[1]):
        ref.check(a, dgamma, off, "dgamma")
