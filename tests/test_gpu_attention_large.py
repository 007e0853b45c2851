"""The kernels of many tiles against the formulas in 64 bits (attention_ref.py, evaluated on the GPU head by head): sequences of several
tiles of keys, whose rows several workgroups share, alone and in company, with and without a prefix, both widths, both masks, groups
that divide a tile and groups that do not.  test_attention_plan.py asserts which kernels the sizes below are given to."""
import pytest
import torch

import attention_ref as ref

pytestmark = pytest.mark.gpu
BF16, F64 = torch.bfloat16, torch.float64

# lengths of the queries, keys before them, heads, channels, causal
LARGE = [
    ([1100], 0, 32, 8, 128, True),                                               # one sequence, its rows in eight pieces
    ([1300], 0, 40, 8, 128, False),
    ([300, 700, 513, 64, 451, 1, 600], 0, 32, 8, 128, True),                     # company, one to three pieces
    ([300, 700, 513, 64, 451, 1, 600, 400, 380, 290, 640], 77, 32, 8, 64, True),
    ([513, 700, 300, 33, 0, 450, 620], 77, 34, 2, 128, True),                    # a group of 17, up to eight pieces
    ([513, 700, 300, 33, 450, 620], 0, 40, 8, 128, False),                       # a group of 5
    ([700, 300, 500, 620, 333, 5, 290, 410, 550, 480], 0, 40, 8, 64, False),
    ([3000], 0, 16, 16, 64, False),                                              # no sharing
    ([900, 20, 3, 500, 100], 300, 24, 8, 128, True),                             # a group of 3, single tiles behind a prefix
    ([2200, 31, 300], 0, 36, 4, 128, True),                                      # a long one in company, a group of 9
]
# the kernels of few tiles over more than 256 keys
FEW = [([700], 0, 2, 2, 64, True), ([310, 290], 40, 6, 2, 128, True), ([400], 0, 4, 1, 64, False)]


@pytest.fixture(scope="module")
def jet():
    import paper_2601_14243_amd as j
    assert torch.cuda.is_available()
    j.lib()
    return j


def _spans(lengths):
    return [sum(lengths[:i]) for i in range(len(lengths) + 1)]


def _inputs(case, seed, std):
    lq, prefix, n_q, n_kv, dim, causal = case
    cu_q, cu_k = _spans(lq), _spans([n + prefix for n in lq])
    gen = torch.Generator(device="cuda").manual_seed(seed)
    normal = lambda rows, heads, s: (torch.randn((rows, heads, dim), generator=gen, device="cuda") * s).to(BF16)
    return (normal(cu_q[-1], n_q, std), normal(cu_k[-1], n_kv, std), normal(cu_k[-1], n_kv, 1.0), normal(cu_q[-1], n_q, 1e-3), cu_q, cu_k)


def _each_head(case, cu_q, cu_k):
    """(rows of q, rows of k, head, head of the keys, mask) of every head of every sequence."""
    _, _, n_q, n_kv, _, causal = case
    for a, b, c, d in zip(cu_q[:-1], cu_q[1:], cu_k[:-1], cu_k[1:]):
        if b > a:
            see = ref.visible(b - a, d - c, causal).cuda()
            for h in range(n_q):
                yield slice(a, b), slice(c, d), h, h // (n_q // n_kv), see


def _run(jet, case, q, k, v, do, cu_q, cu_k):
    kw = dict(cu_q=torch.tensor(cu_q, dtype=torch.int32, device="cuda"), cu_k=torch.tensor(cu_k, dtype=torch.int32, device="cuda"), causal=case[5])
    o, lse = jet.attention_fwd(q, k, v, **kw)
    return o, lse, *jet.attention_bwd(q, k, v, o, lse, do, **kw)


@pytest.mark.parametrize("case", LARGE, ids=lambda c: f"{len(c[0])}x{max(c[0])}+{c[1]}-{c[2]}.{c[3]}.{c[4]}-{c[5]}")
def test_forward_and_backward_of_many_tiles(jet, case):
    q, k, v, do, cu_q, cu_k = _inputs(case, 1, 1.5)
    o, lse, *got = _run(jet, case, q, k, v, do, cu_q, cu_k)
    zero = lambda x: torch.zeros(x.shape, dtype=F64, device="cuda")
    want, tol = [zero(x) for x in (q, k, v)], [zero(x) for x in (q, k, v)]
    for rq, rk, h, g, see in _each_head(case, cu_q, cu_k):
        x = [q[rq, h].to(F64), k[rk, g].to(F64), v[rk, g].to(F64)]
        f = ref.forward(*x, case[4] ** -0.5, see)
        ref.check(o[rq, h], f["o"].cpu(), f["o_tol"].cpu(), f"o {h}")
        ref.check(lse[h, rq], f["lse"].cpu(), f["lse_tol"].cpu(), f"lse {h}")
        grad, t = ref.backward(*x, do[rq, h].to(F64), case[4] ** -0.5, see)
        for into, parts in ((want, grad), (tol, t)):
            into[0][rq, h] = parts[0]
            into[1][rk, g] += parts[1]
            into[2][rk, g] += parts[2]
    for name, a, b, t in zip(("dq", "dk", "dv"), got, want, tol):
        ref.check(a, b.cpu(), (t + ref.BF * (b.abs() + t)).cpu(), name)
    for a, b in zip(got, _run(jet, case, q, k, v, do, cu_q, cu_k)[2:]):
        assert torch.equal(a.view(torch.int16), b.view(torch.int16))


@pytest.mark.parametrize("value", [float("nan"), float("inf")])
@pytest.mark.parametrize("case", [LARGE[2], LARGE[5]], ids=["causal", "all"])
def test_long_neighbours_have_no_influence(jet, case, value):
    """The same as for short ones, on sequences of many tiles: nothing of the neighbours, whatever they hold, changes a bit."""
    q, k, v, do, cu_q, cu_k = _inputs(case, 2, 1.5)
    base = _run(jet, case, q, k, v, do, cu_q, cu_k)
    a, b = cu_q[1], cu_q[2]
    for x in (q, k, v, do):
        x[:a] = value
        x[b:] = value
    for i, (s, t) in enumerate(zip(base, _run(jet, case, q, k, v, do, cu_q, cu_k))):
        s, t = (s[:, a:b], t[:, a:b]) if i == 1 else (s[a:b], t[a:b])
        assert torch.equal(s, t)


@pytest.mark.parametrize("std", [2.5, 4.0])
@pytest.mark.parametrize("case", LARGE[:1] + LARGE[2:5] + FEW, ids=lambda c: f"{len(c[0])}x{max(c[0])}+{c[1]}-{c[2]}.{c[3]}.{c[4]}-{c[5]}")
def test_gradients_of_rows_whose_probability_lies_on_few_keys(jet, case, std):
    """Scores of a large spread, so that most rows have nearly all their probability on one or two of many keys: dp - delta is there a small
    difference of large numbers, and delta has to be better than do o of a rounded o.  attention_ref.peaked_backward counts what is left."""
    q, k, v, do, cu_q, cu_k = _inputs(case, 3, std)
    got = _run(jet, case, q, k, v, do, cu_q, cu_k)[2:4]
    want, tol = [[torch.zeros(x.shape, dtype=F64, device="cuda") for x in (q, k)] for _ in range(2)]
    for rq, rk, h, g, see in _each_head(case, cu_q, cu_k):
        grad, t = ref.peaked_backward(q[rq, h].to(F64), k[rk, g].to(F64), v[rk, g].to(F64), do[rq, h].to(F64), case[4] ** -0.5, see)
        for into, parts in ((want, grad), (tol, t)):
            into[0][rq, h] = parts[0]
            into[1][rk, g] += parts[1]
    for name, a, b, t in zip(("dq", "dk"), got, want, tol):
        ref.check(a, b.cpu(), (t + ref.BF * (b.abs() + t)).cpu(), name)
    # dk has delta in 32 bits: two independent roundings, uniform within half a step, as for rows that see few keys
    b = want[1]
    assert (got[1].to(F64) - b).norm() <= 2 ** 0.5 * torch.finfo(BF16).eps / 2 / 3 ** 0.5 * b.norm()


@pytest.mark.parametrize("case", [([700], 33, 2, 2, 128, True), ([1600], 33, 16, 16, 128, True), ([900], 7, 24, 8, 64, True), ([2000], 0, 32, 8, 64, True)],
                         ids=lambda c: f"{c[0][0]}+{c[1]}-{c[2]}.{c[3]}.{c[4]}")
def test_how_far_what_is_not_finite_reaches(jet, case):
    """A value, key, query or output gradient that is infinite: rows (keys) that neither see it nor lie within a tile of one that does keep
    their bytes, 94 positions for the forward pass and 62 for the gradients being the most that tiles can put between them."""
    lq, prefix, n_q, n_kv, dim, _ = case
    n, group = lq[0], n_q // n_kv
    q, k, v, do, cu_q, cu_k = _inputs(case, 4, 1.5)
    kw = dict(cu_q=torch.tensor(cu_q, dtype=torch.int32, device="cuda"), cu_k=torch.tensor(cu_k, dtype=torch.int32, device="cuda"))
    o, lse = jet.attention_fwd(q, k, v, **kw)
    dq, dk, dv = jet.attention_bwd(q, k, v, o, lse, do, **kw)
    same = lambda a, b: torch.equal(a.contiguous().view(torch.int16), b.contiguous().view(torch.int16))
    for at in (prefix + 127, prefix + 128, prefix + 300, prefix + n - 1):                  # the last key of row at - prefix
        heads = slice(group, 2 * group)                                                    # of key head 1
        y = v.clone()
        y[at, 1, 3] = float("inf")
        got, got_lse = jet.attention_fwd(q, k, y, **kw)
        assert torch.equal(got_lse, lse)
        assert same(got[:at - prefix - 94], o[:at - prefix - 94]) and not got[at - prefix:, heads].isfinite().all()
        assert same(got[:, :group], o[:, :group])                                          # the other heads keep theirs
        y = k.clone()
        y[at, 1, 3] = float("inf")
        got, got_lse = jet.attention_fwd(q, y, v, **kw)
        assert got[:at - prefix].isfinite().all() and got_lse[:, :at - prefix].isfinite().all()      # its score is left out
        assert same(got[:, :group], o[:, :group]) and torch.equal(got_lse[:group], lse[:group])
        got = jet.attention_bwd(q, y, v, o, lse, do, **kw)[0]
        assert same(got[:at - prefix - 62], dq[:at - prefix - 62]) and same(got[:, :group], dq[:, :group])
        for i in range(2):
            x = [q.clone(), do.clone()]
            x[i][at - prefix, group, 3] = float("inf")
            a, b, c = jet.attention_bwd(x[0], k, v, o, lse, x[1], **kw)
            assert same(b[at + 63:], dk[at + 63:]) and same(c[at + 63:], dv[at + 63:])
            assert same(a[:, :group], dq[:, :group]) and same(b[:, 0], dk[:, 0]) and same(c[:, 0], dv[:, 0])


@pytest.mark.parametrize("case", [LARGE[0], LARGE[4], LARGE[6], FEW[1]], ids=lambda c: f"{len(c[0])}x{max(c[0])}+{c[1]}-{c[2]}.{c[3]}.{c[4]}-{c[5]}")
def test_gradients_of_a_few_rows_whose_probability_lies_on_few_keys(jet, case):
    """Flat rows but for single ones, so that one wave of a tile goes over its keys again and the others only copy; that those have a
    correction to make is seen from do o of the o that the forward pass returned."""
    q, k, v, do, cu_q, cu_k = _inputs(case, 5, 0.7)
    peaked = [(t, t % q.shape[1]) for t in range(301, q.shape[0], 211)] + [(q.shape[0] - 1, q.shape[1] - 1)]
    for t, h in peaked:
        q[t, h] *= 24
    o, lse, dq, dk, _ = _run(jet, case, q, k, v, do, cu_q, cu_k)
    want, tol = [[torch.zeros(x.shape, dtype=F64, device="cuda") for x in (q, k)] for _ in range(2)]
    beyond = 0
    for rq, rk, h, g, see in _each_head(case, cu_q, cu_k):
        x = [q[rq, h].to(F64), k[rk, g].to(F64), v[rk, g].to(F64), do[rq, h].to(F64)]
        grad, t = ref.peaked_backward(*x, case[4] ** -0.5, see)
        for into, parts in ((want, grad), (tol, t)):
            into[0][rq, h] = parts[0]
            into[1][rk, g] += parts[1]
        rows = [t - rq.start for t, head in peaked if head == h and rq.start <= t < rq.stop]
        p = torch.softmax((x[0][rows] @ x[1].T * case[4] ** -0.5).masked_fill(~see[rows], float("-inf")), dim=1)
        dp = x[3][rows] @ x[2].T
        ds = p * (dp - (p * dp).sum(dim=1, keepdim=True))
        e = (p * dp).sum(dim=1) - (x[3][rows] * o[rq, h][rows].to(F64)).sum(dim=1)
        beyond += int((e.abs() > 2 * ref.BF * ds.abs().sum(dim=1)).sum())
    assert beyond > 0
    for name, a, b, t in zip(("dq", "dk"), (dq, dk), want, tol):
        ref.check(a, b.cpu(), (t + ref.BF * (b.abs() + t)).cpu(), name)
