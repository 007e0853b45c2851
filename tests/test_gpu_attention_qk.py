"""qk_norm_rope and its gradient on more tokens than test_gpu_attention.py has: four heads to a team of lanes, head counts that four does and
does not divide.  test_attention_plan.py asserts that the sizes below are given to those kernels."""
import pytest
import torch

import attention_ref as ref

pytestmark = pytest.mark.gpu
BF16 = torch.bfloat16
ROWS = 512

MANY = [(5700, 5, 3, 128, True), (11200, 9, 2, 64, True), (8300, 6, 1, 128, False), (10001, 14, 7, 64, False), (1700, 32, 8, 128, True)]   # tokens, heads, channels, norm
MANY_BWD = [(5700, 5, 3, 128, True), (11200, 9, 2, 64, True), (8300, 6, 1, 128, False), (10001, 14, 7, 64, False), (1000, 32, 8, 128, True)]
MANY_KEPT = [(4200, 5, 3, 128, 48, False), (4200, 5, 3, 128, 16, True), (8200, 9, 2, 64, 64, True), (8200, 6, 1, 64, 16, False)]            # ..., page, E4M3


@pytest.fixture(scope="module")
def jet():
    import paper_2601_14243_amd as j
    assert torch.cuda.is_available()
    j.lib()
    return j


def _case(T, n_q, n_kv, dim, norm, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    normal = lambda shape, std: (torch.randn(shape, generator=gen, device="cuda") * std).to(BF16)
    inv = 1e4 ** (-torch.arange(0, dim, 2, dtype=torch.float64, device="cuda") / dim)
    ang = torch.arange(ROWS, dtype=torch.float64, device="cuda")[:, None] * inv
    table = torch.cat([ang.cos(), ang.sin()], dim=1).float()
    pos = torch.randint(0, ROWS, (T,), generator=gen, device="cuda").int()
    gam = [1 + normal((dim,), 0.2) for _ in range(2)] if norm else [None, None]
    return normal((T, n_q + 2 * n_kv, dim), 1.5), table, pos, gam, [normal((T, h, dim), 1e-3) for h in (n_q, n_kv)]


def _check(got, want, tol, name):
    ref.check(got, want.cpu(), tol.cpu(), name)


@pytest.mark.parametrize("T,n_q,n_kv,dim,norm", MANY)
def test_norm_and_rotation_of_many_tokens(jet, T, n_q, n_kv, dim, norm):
    x, table, pos, gam, _ = _case(T, n_q, n_kv, dim, norm, 1)
    wide = torch.zeros((T, (n_q + 2 * n_kv) * dim + 24), dtype=BF16, device="cuda")
    wide[:, :-24] = x.flatten(1)
    got = jet.qk_norm_rope(wide[:, :-24], n_q, n_kv, table, pos, *gam, 1e-6)
    for part, g, y, name in zip(x.double().split([n_q, n_kv, n_kv], dim=1), gam, got, "qk"):
        want, tol = ref.norm_rope(part, None if g is None else g.double(), table.double(), pos.long(), 1e-6)
        _check(y, want, tol, name)


@pytest.mark.parametrize("T,n_q,n_kv,dim,norm", MANY_BWD)
def test_gradient_of_norm_and_rotation_of_many_tokens(jet, T, n_q, n_kv, dim, norm):
    x, table, pos, gam, dy = _case(T, n_q, n_kv, dim, norm, 2)
    dx, *dgam = jet.qk_norm_rope_bwd(*dy, x.flatten(1), table, pos, *gam, 1e-6)
    parts, got = x.double().split([n_q, n_kv, n_kv], dim=1), dx.view(T, n_q + n_kv, dim).split([n_q, n_kv], dim=1)
    for i, name in enumerate("qk"):
        g = None if gam[i] is None else gam[i].double()
        want, tol, dg, dg_tol = ref.norm_rope_backward(dy[i].double(), parts[i], g, table.double(), pos.long(), 1e-6)
        _check(got[i], want, tol, "d" + name)
        if norm:
            _check(dgam[i], dg, dg_tol, "dgamma_" + name)
        else:
            assert dgam[i] is None
    out = torch.full((T, (n_q + n_kv) * dim + 40), 5.0, dtype=BF16, device="cuda")
    jet.qk_norm_rope_bwd(*dy, x.flatten(1), table, pos, *gam, 1e-6, out=out)
    assert torch.equal(out[:, :dx.shape[1]], dx) and (out[:, dx.shape[1]:] == 5).all()


@pytest.mark.parametrize("T,n_q,n_kv,dim,page,fp8", MANY_KEPT)
def test_many_keys_and_values_go_to_their_slots(jet, T, n_q, n_kv, dim, page, fp8):
    x, table, pos, gam, _ = _case(T, n_q, n_kv, dim, True, 3)
    n_pages = T // page + 3
    slots = torch.randperm(n_pages * page, generator=torch.Generator().manual_seed(4))[:T].cuda()
    slots[5], slots[T - 1] = -1, n_pages * page              # not kept
    keep = torch.ones(T, dtype=torch.bool, device="cuda")
    keep[5] = keep[T - 1] = False
    shape = (n_pages, n_kv, page, dim)
    kv = [torch.full(shape, 9, dtype=torch.uint8 if fp8 else BF16, device="cuda") for _ in range(2)]
    sc = [torch.full(shape[:3], -1.0, device="cuda") for _ in range(2)] if fp8 else [None, None]
    q, k = jet.qk_norm_rope(x.flatten(1), n_q, n_kv, table, pos, *gam, cache=jet.KvCache(*kv, *sc), slots=slots)
    q2, k2 = jet.qk_norm_rope(x.flatten(1), n_q, n_kv, table, pos, *gam)
    assert torch.equal(q, q2) and torch.equal(k, k2)
    at = slots[keep]
    for c, s, new in zip(kv, sc, (k, x[:, n_q + n_kv:])):
        rows = c.transpose(1, 2).reshape(n_pages * page, n_kv, dim)
        rest = torch.ones(n_pages * page, dtype=torch.bool, device="cuda")
        rest[at] = False
        assert (rows[rest] == 9).all()
        new = new[keep]
        if not fp8:
            assert torch.equal(rows[at], new)
            continue
        new = new.float().cpu()                              # a GPU divides by a constant as a product with its inverse
        top = new.abs().amax(dim=2)
        S = torch.where(top == 0, torch.ones_like(top), top / 448)
        scales = s.transpose(1, 2).reshape(n_pages * page, n_kv)
        assert (scales[rest] == -1).all() and torch.equal(scales[at].cpu(), S)
        assert torch.equal(rows[at].cpu(), (new / S[..., None]).to(torch.float8_e4m3fn).view(torch.uint8))


@pytest.mark.parametrize("T,n_q,n_kv,dim,norm", MANY)
def test_a_token_gets_the_same_bytes_alone_and_among_many(jet, T, n_q, n_kv, dim, norm):
    """Rollout and training: one head to a team and four."""
    x, table, pos, gam, dy = _case(T, n_q, n_kv, dim, norm, 5)
    many = jet.qk_norm_rope(x.flatten(1), n_q, n_kv, table, pos, *gam)
    dx = jet.qk_norm_rope_bwd(*dy, x.flatten(1), table, pos, *gam)[0]
    for a, b in ((0, 1), (T // 2, T // 2 + 37), (T - 3, T)):
        few = jet.qk_norm_rope(x[a:b].flatten(1), n_q, n_kv, table, pos[a:b].contiguous(), *gam)
        assert all(torch.equal(s[a:b].view(torch.int16), t.view(torch.int16)) for s, t in zip(many, few))
        one = jet.qk_norm_rope_bwd(dy[0][a:b], dy[1][a:b], x[a:b].flatten(1), table, pos[a:b].contiguous(), *gam)[0]
        assert torch.equal(dx[a:b].view(torch.int16), one.view(torch.int16))
