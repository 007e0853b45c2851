"""qk_norm_rope, attention_fwd, attention_bwd and attention_decode against their formulas in 64 bits (attention_ref.py), within bounds
that count roundings."""
import math

import pytest
import torch

import attention_ref as ref

pytestmark = pytest.mark.gpu
BF16 = torch.bfloat16


@pytest.fixture(scope="module")
def jet():
    import paper_2601_14243_amd as j
    assert torch.cuda.is_available()
    j.lib()
    return j


def _normal(seed, shape, std=1.0):
    return (torch.randn(shape, generator=torch.Generator().manual_seed(seed)) * std).to(BF16)


def _cu(lengths):
    return [sum(lengths[:i]) for i in range(len(lengths) + 1)]


def _i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


# lengths of the queries, of the keys (None: the same), heads, channels, causal
PACKED = [
    ([1], None, 4, 2, 128, True),                           # one token
    ([37], None, 8, 2, 128, True),
    ([1, 0, 5, 64, 0, 65, 130, 3], None, 6, 1, 64, True),   # empty sequences, a group of 6
    ([128, 32, 31, 33], None, 4, 4, 128, True),             # tile edges, no sharing
    ([257], None, 5, 1, 128, True),                         # a group that divides no tile
    ([17, 40], [300, 40], 8, 2, 64, True),                  # keys that came before the queries
    ([1, 1, 2], [129, 64, 1], 12, 2, 128, True),            # single tokens behind long prefixes
    ([50, 70], [20, 100], 4, 2, 128, True),                 # first rows that see no key
    ([9, 30, 4], [0, 64, 7], 4, 2, 64, True),               # a sequence without keys
    ([0, 30], [64, 30], 4, 2, 128, True),                   # keys without queries
    ([100, 1, 63], [63, 200, 1], 8, 8, 64, False),
    ([45, 200], None, 32, 8, 128, False),
    ([3, 90], None, 34, 2, 64, True),                       # a group of 17
    ([700], None, 2, 2, 64, True),
]


def _inputs(case, seed=0, std=1.5):
    lq, lk, n_q, n_kv, dim, causal = case
    lk = lq if lk is None else lk
    cu_q, cu_k = _cu(lq), _cu(lk)
    q = _normal(seed, (cu_q[-1], n_q, dim), std)
    k = _normal(seed + 1, (cu_k[-1], n_kv, dim), std)
    v = _normal(seed + 2, (cu_k[-1], n_kv, dim))
    do = _normal(seed + 3, (cu_q[-1], n_q, dim), 1e-3)
    return q, k, v, do, cu_q, cu_k, causal, dim ** -0.5


# more sequences than a wave has lanes, and the most that still fit them
PACKED += [([i * 37 % 23 for i in range(n)], None, 4, 2, 64, True) for n in (61, 62, 190)]


@pytest.mark.parametrize("case", PACKED, ids=lambda c: f"{c[0][:8]}x{len(c[0])}-{c[1]}-{c[2]}.{c[3]}.{c[4]}-{c[5]}")
def test_forward_and_backward(jet, case):
    q, k, v, do, cu_q, cu_k, causal, scale = _inputs(case)
    o, lse, o_tol, lse_tol = ref.packed_forward(q, k, v, cu_q, cu_k, scale, causal)
    g, tol = ref.packed_backward(q, k, v, do, cu_q, cu_k, scale, causal)
    dev = [x.cuda() for x in (q, k, v, do)]
    kw = dict(cu_q=_i32(cu_q), cu_k=_i32(cu_k), causal=causal)
    got_o, got_lse = jet.attention_fwd(*dev[:3], **kw)
    ref.check(got_o, o, o_tol, "o")
    ref.check(got_lse, lse, lse_tol, "lse")
    got = jet.attention_bwd(*dev[:3], got_o, got_lse, dev[3], **kw)
    for name, a, b, t in zip(("dq", "dk", "dv"), got, g, tol):
        ref.check(a, b, t, name)
    again = jet.attention_bwd(*dev[:3], got_o, got_lse, dev[3], **kw)
    for a, b in zip(got, again):
        assert torch.equal(a.view(torch.int16), b.view(torch.int16))


def test_slices_of_wider_rows_and_outputs_in_them(jet):
    """q, k and v where a projection left them, gradients where its backward pass wants them."""
    n_q, n_kv, dim, lens = 8, 2, 128, [70, 3, 129]
    cu = _cu(lens)
    wide = _normal(5, (cu[-1], n_q + 2 * n_kv, dim), 1.2).cuda()
    q, k, v = wide[:, :n_q], wide[:, n_q:n_q + n_kv], wide[:, n_q + n_kv:]
    do = _normal(6, (cu[-1], n_q, dim)).cuda()
    o, lse = jet.attention_fwd(q, k, v, cu_q=_i32(cu))
    o2, lse2 = jet.attention_fwd(q.contiguous(), k.contiguous(), v.contiguous(), cu_q=_i32(cu))
    assert torch.equal(o, o2) and torch.equal(lse, lse2)
    grad = torch.full_like(wide, 7.0)
    out = (grad[:, :n_q], grad[:, n_q:n_q + n_kv], grad[:, n_q + n_kv:])
    res = jet.attention_bwd(q, k, v, o, lse, do, cu_q=_i32(cu), out=out)
    assert all(a is b for a, b in zip(res, out))
    want = jet.attention_bwd(q.contiguous(), k.contiguous(), v.contiguous(), o, lse, do, cu_q=_i32(cu))
    assert torch.equal(grad, torch.cat(want, dim=1))


@pytest.mark.parametrize("value", [math.nan, math.inf, -torch.finfo(BF16).max])
def test_other_sequences_have_no_influence(jet, value):
    """Keys, values, queries and gradients of the neighbours hold `value`: the middle sequence's results do not change by a bit."""
    n_q, n_kv, dim, lens = 6, 2, 64, [40, 75, 33]
    cu = _cu(lens)
    a, b = cu[1], cu[2]
    x = [_normal(10 + i, (cu[-1], h, dim)).cuda() for i, h in enumerate((n_q, n_kv, n_kv, n_q))]
    y = [t.clone() for t in x]
    for t in y:
        t[:a] = value
        t[b:] = value
    kw = dict(cu_q=_i32(cu))
    o, lse = jet.attention_fwd(*x[:3], **kw)
    o2, lse2 = jet.attention_fwd(*y[:3], **kw)
    assert torch.equal(o[a:b], o2[a:b]) and torch.equal(lse[:, a:b], lse2[:, a:b])
    for s, t in zip(jet.attention_bwd(*x[:3], o, lse, x[3], **kw), jet.attention_bwd(*y[:3], o2, lse2, y[3], **kw)):
        assert torch.equal(s[a:b], t[a:b])


def test_rows_of_no_sequence(jet):
    """Rows behind the last boundary (and in front of the first) have no keys: o = 0, lse = -inf, no gradients."""
    n_q, n_kv, dim = 4, 2, 64
    x = [_normal(20 + i, (200, h, dim)).cuda() for i, h in enumerate((n_q, n_kv, n_kv, n_q))]
    kw = dict(cu_q=_i32([10, 60, 150]))
    o, lse = jet.attention_fwd(*x[:3], **kw)
    g = jet.attention_bwd(*x[:3], o, lse, x[3], **kw)
    rest = torch.ones(200, dtype=torch.bool)
    rest[10:150] = False
    assert not o[rest].any() and (lse[:, rest] == -math.inf).all() and all(not t[rest].any() for t in g)
    inner = [torch.cat([t[10:], t[:10]]) for t in x]         # the same sizes, on which the order of the sums depends
    kw = dict(cu_q=_i32([0, 50, 140]))
    o2, lse2 = jet.attention_fwd(*inner[:3], **kw)
    assert torch.equal(o[10:150], o2[:140]) and torch.equal(lse[:, 10:150], lse2[:, :140])
    for s, t in zip(g, jet.attention_bwd(*inner[:3], o2, lse2, inner[3], **kw)):
        assert torch.equal(s[10:150], t[:140])


@pytest.mark.parametrize("cu", [[-50, 40, 1000], [90, 20, 150], [0, 400, 100], [150, 0, 0]])
def test_wrong_boundaries_stay_inside_the_arrays(jet, cu):
    """Boundaries that do not ascend or leave the array are cut to it: no answer is promised, no access outside and no wait."""
    n_q, n_kv, dim = 4, 2, 64
    guard = 64
    x = [_normal(30 + i, (150, h, dim)).cuda() for i, h in enumerate((n_q, n_kv, n_kv, n_q))]
    o, lse = jet.attention_fwd(*x[:3], cu_q=_i32(cu))
    buf = [torch.full((150 + 2 * guard, h, dim), 3.0, dtype=BF16, device="cuda") for h in (n_q, n_kv, n_kv)]
    jet.attention_bwd(*x[:3], o, lse, x[3], cu_q=_i32(cu), out=tuple(t[guard:guard + 150] for t in buf))
    torch.cuda.synchronize()
    for t in buf:
        assert (t[:guard] == 3).all() and (t[guard + 150:] == 3).all()


def test_scale_and_large_scores(jet):
    """A scale of one's own, and scores whose exponentials overflow binary32 without the running maximum."""
    q, k, v, do, cu_q, cu_k, causal, _ = _inputs(([90, 20], None, 4, 2, 64, True), seed=40, std=12.0)
    o, lse, o_tol, lse_tol = ref.packed_forward(q, k, v, cu_q, cu_k, 0.5, causal)
    assert lse.max() > 200
    got_o, got_lse = jet.attention_fwd(q.cuda(), k.cuda(), v.cuda(), cu_q=_i32(cu_q), scale=0.5)
    ref.check(got_o, o, o_tol, "o")
    ref.check(got_lse, lse, lse_tol, "lse")


@pytest.mark.parametrize("lq, prefix, n_q, n_kv, dim, short", [
    ([2] * 5, 0, 8, 8, 64, 5), ([1] * 19, 1, 8, 8, 64, 19), ([2, 3, 4] * 40, 0, 8, 2, 128, 120),
    ([2] * 20 + [900], 0, 4, 2, 64, 20), ([3, 2] * 10 + [900], 0, 8, 2, 128, 20)])          # short ones in the company of a long one
def test_gradients_of_rows_that_see_few_keys(jet, lq, prefix, n_q, n_kv, dim, short):
    """dp - delta is there a small difference of large numbers.  What a gradient rounds to bf16 is ds for the products and the result: two
    independent errors, uniform within half a step, at most eps / 2 / sqrt(3) of the value in the 2-norm.  The rest is in 32 bits."""
    q, k, v, do, cu_q, cu_k, causal, scale = _inputs((lq, [n + prefix for n in lq], n_q, n_kv, dim, True), seed=90, std=1.0)
    g, _ = ref.packed_backward(q, k, v, do, cu_q, cu_k, scale, causal)
    kw = dict(cu_q=_i32(cu_q), cu_k=_i32(cu_k))
    o, lse = jet.attention_fwd(q.cuda(), k.cuda(), v.cuda(), **kw)
    got = jet.attention_bwd(q.cuda(), k.cuda(), v.cuda(), o, lse, do.cuda(), **kw)
    for name, a, b, rows in (("dq", got[0], g[0], cu_q[short]), ("dk", got[1], g[1], cu_k[short])):
        a, b = a[:rows].cpu().double(), b[:rows]
        assert (a - b).norm() <= 2 ** 0.5 * torch.finfo(BF16).eps / 2 / 3 ** 0.5 * b.norm(), (name, ((a - b).norm() / b.norm()).item())


def test_gradient_against_differences(jet):
    """Directional derivatives of sum(o do), differences of the 64-bit forward pass, against the kernels' gradients."""
    q, k, v, do, cu_q, cu_k, causal, scale = _inputs(([20, 45], [33, 45], 4, 2, 64, True), seed=50, std=1.0)
    kw = dict(cu_q=_i32(cu_q), cu_k=_i32(cu_k))
    o, lse = jet.attention_fwd(q.cuda(), k.cuda(), v.cuda(), **kw)
    got = jet.attention_bwd(q.cuda(), k.cuda(), v.cuda(), o, lse, do.cuda(), **kw)
    _, tol = ref.packed_backward(q, k, v, do, cu_q, cu_k, scale, causal)
    x = [t.double() for t in (q, k, v)]
    loss = lambda y: (ref.packed_forward(*y, cu_q, cu_k, scale, causal)[0] * do.double()).sum()
    for i in range(3):
        d = torch.randn(x[i].shape, generator=torch.Generator().manual_seed(60 + i), dtype=torch.float64)
        h = 1e-4
        up, down = list(x), list(x)
        up[i], down[i] = x[i] + h * d, x[i] - h * d
        slope = (loss(up) - loss(down)) / (2 * h)
        mine = (got[i].cpu().double() * d).sum()
        # the gradient's own bound along d, and the third derivative's share of a central difference
        assert abs(slope - mine) <= (tol[i] * d.abs()).sum() + 1e-4 * abs(slope) + 1e-9, (i, slope, mine)


# ------------------------------------------------------------- norm and rotation

def _table(dim, rows=512):
    inv = 1e4 ** (-torch.arange(0, dim, 2, dtype=torch.float64) / dim)
    ang = torch.arange(rows, dtype=torch.float64)[:, None] * inv
    return torch.cat([ang.cos(), ang.sin()], dim=1).float()


QK = [(1, 32, 8, 128, True), (1, 6, 1, 64, False), (3, 5, 3, 128, True), (130, 8, 2, 64, True), (77, 9, 2, 128, False), (1500, 16, 2, 64, True),
      (701, 32, 8, 128, True)]


@pytest.mark.parametrize("T,n_q,n_kv,dim,norm", QK)
def test_norm_and_rotation(jet, T, n_q, n_kv, dim, norm):
    x = _normal(70, (T, n_q + 2 * n_kv, dim), 1.5)
    x[0, 0] = 0                                              # a head of zeros: r = eps^-1/2
    table, gen = _table(dim), torch.Generator().manual_seed(71)
    pos = torch.randint(0, 512, (T,), generator=gen).int()
    gam = [(1 + 0.2 * torch.randn(dim, generator=gen)).to(BF16) for _ in range(2)] if norm else [None, None]
    dev = lambda t: None if t is None else t.cuda()
    wide = torch.zeros((T, (n_q + 2 * n_kv) * dim + 24), dtype=BF16)
    wide[:, :-24] = x.flatten(1)
    rows = wide.cuda()[:, :-24]                              # rows that lie further apart
    got = jet.qk_norm_rope(rows, n_q, n_kv, table.cuda(), pos.cuda(), dev(gam[0]), dev(gam[1]), 1e-6)
    dy = [_normal(72 + i, (T, h, dim), 1e-3) for i, h in enumerate((n_q, n_kv))]
    dx, *dgam = jet.qk_norm_rope_bwd(dy[0].cuda(), dy[1].cuda(), rows, table.cuda(), pos.cuda(), dev(gam[0]), dev(gam[1]), 1e-6)
    parts = x.double().split([n_q, n_kv, n_kv], dim=1)
    dx = dx.view(T, n_q + n_kv, dim).split([n_q, n_kv], dim=1)
    for i, name in enumerate("qk"):
        g = None if gam[i] is None else gam[i].double()
        y, tol = ref.norm_rope(parts[i], g, table.double(), pos.long(), 1e-6)
        ref.check(got[i], y, tol, name)
        want, tol, dg, dg_tol = ref.norm_rope_backward(dy[i].double(), parts[i], g, table.double(), pos.long(), 1e-6)
        ref.check(dx[i], want, tol, "d" + name)
        if norm:
            ref.check(dgam[i], dg, dg_tol, "dgamma_" + name)
        else:
            assert dgam[i] is None


def test_rotation_gradient_into_the_projections_gradient(jet):
    T, n_q, n_kv, dim = 9, 4, 2, 64
    x = _normal(80, (T, (n_q + 2 * n_kv) * dim)).cuda()
    gam = [_normal(81 + i, (dim,)).cuda() for i in range(2)]
    dq, dk = _normal(83, (T, n_q, dim)).cuda(), _normal(84, (T, n_kv, dim)).cuda()
    pos = torch.arange(T, dtype=torch.int32, device="cuda")
    want, *dg = jet.qk_norm_rope_bwd(dq, dk, x, _table(dim).cuda(), pos, *gam)
    out = torch.full_like(x, 5.0)
    got, *dg2 = jet.qk_norm_rope_bwd(dq, dk, x, _table(dim).cuda(), pos, *gam, out=out)
    assert got is out and torch.equal(out[:, :want.shape[1]], want) and (out[:, want.shape[1]:] == 5).all()
    assert all(torch.equal(a, b) for a, b in zip(dg, dg2))


def test_a_position_outside_the_table_gives_nan(jet):
    T, n_q, n_kv, dim = 6, 4, 2, 64
    x = _normal(85, (T, (n_q + 2 * n_kv) * dim)).cuda()
    pos = torch.tensor([0, 511, 512, -1, 2 ** 31 - 1, 5], dtype=torch.int32, device="cuda")
    q, k = jet.qk_norm_rope(x, n_q, n_kv, _table(dim).cuda(), pos)
    bad = torch.tensor([False, False, True, True, True, False])
    for t in (q, k):
        assert t[bad].isnan().all() and t[~bad].isfinite().all()


@pytest.mark.parametrize("T,page,dim,fp8", [(1, 16, 128, False), (50, 16, 64, False), (50, 64, 128, True), (300, 48, 64, True), (700, 128, 128, False)])
def test_keys_and_values_go_to_their_slots(jet, T, page, dim, fp8):
    n_q, n_kv, n_pages = 4, 2, T // page + 3
    x = _normal(90, (T, n_q + 2 * n_kv, dim), 1.5)
    x[0, n_q + n_kv] = 0                                     # a value head of zeros: scale 1
    gen = torch.Generator().manual_seed(91)
    slots = torch.randperm(n_pages * page, generator=gen)[:T]
    keep = torch.ones(T, dtype=torch.bool)
    if T > 4:
        slots[3], slots[1] = -1, n_pages * page              # not kept
        keep[3] = keep[1] = False
    pos = torch.randint(0, 512, (T,), generator=gen).int().cuda()
    shape = (n_pages, n_kv, page, dim)
    kv = [torch.full(shape, 9, dtype=torch.uint8 if fp8 else BF16, device="cuda") for _ in range(2)]
    sc = [torch.full(shape[:3], -1.0, device="cuda") for _ in range(2)] if fp8 else [None, None]
    cache = jet.KvCache(*kv, *sc)
    q, k = jet.qk_norm_rope(x.flatten(1).cuda(), n_q, n_kv, _table(dim).cuda(), pos, cache=cache, slots=slots.cuda())
    q2, k2 = jet.qk_norm_rope(x.flatten(1).cuda(), n_q, n_kv, _table(dim).cuda(), pos)
    assert torch.equal(q, q2) and torch.equal(k, k2)
    touched = torch.zeros((n_pages, page), dtype=torch.bool)
    for c, s, new in zip(kv, sc, (k.cpu(), x[:, n_q + n_kv:])):
        c = c.cpu()
        for t in range(T):
            if not keep[t]:
                continue
            p, r = int(slots[t]) // page, int(slots[t]) % page
            touched[p, r] = True
            if fp8:                                          # the row quantizer's scale and codes of the bf16 values
                top = new[t].float().abs().amax(dim=1)
                S = torch.where(top == 0, torch.ones(()), top / 448)
                assert torch.equal(s[p, :, r].cpu(), S)
                assert torch.equal(c[p, :, r], (new[t].float() / S[:, None]).to(torch.float8_e4m3fn).view(torch.uint8))
            else:
                assert torch.equal(c[p, :, r], new[t])
        rest = c.transpose(1, 2)[~touched]
        assert (rest == 9).all()
        if fp8:
            assert (s.cpu().transpose(1, 2)[~touched] == -1).all()


# ------------------------------------------------------------------------ decode

# lengths, heads, channels, page, spare columns of the page table
DECODE = [
    ([1], 8, 2, 128, 16, 0),
    ([700], 32, 8, 128, 64, 0),
    ([0, 1, 15, 16, 17, 31, 32, 33, 127, 128, 129], 4, 2, 64, 16, 3),
    ([300, 5, 64], 5, 1, 128, 64, 1),
    ([1000, 999], 40, 8, 128, 128, 40),
    ([200, 1, 77], 6, 1, 64, 48, 0),
    ([130, 250], 34, 2, 64, 32, 0),                          # a group of 17: two blocks of query heads
    ([2500, 40, 0], 8, 8, 64, 32, 200),
    ([33] * 40, 16, 16, 128, 16, 0),
]


def _paged(jet, lengths, n_kv, dim, page, spare, fp8, seed=100):
    gen = torch.Generator().manual_seed(seed)
    need = [-(-n // page) for n in lengths]
    n_pages = sum(need) + 3
    order = torch.randperm(n_pages, generator=gen).int()
    pages = torch.full((len(lengths), max(max(need), 1) + spare), -7, dtype=torch.int32)   # entries that no length needs
    at = 0
    for i, n in enumerate(need):
        pages[i, :n] = order[at:at + n]
        at += n
    x = [torch.randn((n_pages, n_kv, page, dim), generator=gen) * s for s in (1.5, 1.0)]
    held = torch.zeros((n_pages, page), dtype=torch.bool)
    for b, n in enumerate(lengths):
        for j in range(n):
            held[pages[b, j // page], j % page] = True
    held = held[:, None, :].expand(n_pages, n_kv, page)
    if fp8:
        sc = [t.abs().amax(dim=3) / 448 for t in x]
        x = [(t / s[..., None]).to(torch.float8_e4m3fn).view(torch.uint8) for t, s in zip(x, sc)]
        x = [torch.where(held[..., None], t, torch.full_like(t, 0x7F)) for t in x]      # NaN wherever no key is
        sc = [torch.where(held, s, torch.full_like(s, math.nan)) for s in sc]
    else:
        sc = [None, None]
        x = [torch.where(held[..., None], t, torch.full_like(t, math.nan)).to(BF16) for t in x]
    cache = jet.KvCache(x[0].cuda(), x[1].cuda(), *(None if s is None else s.cuda() for s in sc))
    return cache, x, sc, pages


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("lengths,n_q,n_kv,dim,page,spare", DECODE)
def test_decode(jet, lengths, n_q, n_kv, dim, page, spare, fp8):
    cache, x, sc, pages = _paged(jet, lengths, n_kv, dim, page, spare, fp8)
    q = _normal(101, (len(lengths), n_q, dim), 1.5)
    want, tol = ref.decode(q, *x, *sc, pages, lengths, dim ** -0.5)
    got = jet.attention_decode(q.cuda(), cache, pages.cuda(), _i32(lengths))
    ref.check(got, want, tol, "o")
    assert torch.equal(got, jet.attention_decode(q.cuda(), cache, pages.cuda(), _i32(lengths)))
    wide = torch.zeros((len(lengths), n_q + 3, dim), dtype=BF16)
    wide[:, :n_q] = q
    assert torch.equal(got, jet.attention_decode(wide.cuda()[:, :n_q], cache, pages.cuda(), _i32(lengths)))


@pytest.mark.parametrize("fp8", [False, True])
def test_decode_refuses_bad_pages_with_nan(jet, fp8):
    lengths = [40, 300, 20, 64, -5]
    cache, x, sc, pages = _paged(jet, [40, 300, 20, 64, 0], 2, 64, 16, 0, fp8)
    good = jet.attention_decode(_normal(102, (5, 4, 64)).cuda(), cache, pages.cuda(), _i32(lengths))
    assert good.isfinite().all() and not good[4].any()
    pages[0, 1] = cache.n_pages                              # one past the last
    pages[2, 0] = -1
    lengths[3] = pages.shape[1] * 16 + 1                     # longer than its row of the table
    got = jet.attention_decode(_normal(102, (5, 4, 64)).cuda(), cache, pages.cuda(), _i32(lengths))
    for b in (0, 2, 3):
        assert got[b].isnan().all()
    assert torch.equal(got[1], good[1]) and not got[4].any()


# ------------------------------------------------------------- both host paths

class _Declines:
    def __getattr__(self, name):
        return lambda *a: None


def test_native_and_python_path_agree(jet, monkeypatch):
    from paper_2601_14243_amd import binding as b
    T, n_q, n_kv, dim = 50, 4, 2, 64
    x, table = _normal(200, (T, (n_q + 2 * n_kv) * dim)).cuda(), _table(dim).cuda()
    pos, slots = torch.arange(T, dtype=torch.int32, device="cuda"), torch.arange(T, device="cuda")
    gam = [_normal(201 + i, (dim,)).cuda() for i in range(2)]
    q, k, v, do = (_normal(210 + i, (T, h, dim)).cuda() for i, h in enumerate((n_q, n_kv, n_kv, n_q)))
    cu, lens = _i32([0, 20, T]), _i32([40, 3])
    pages = _i32([[0, 1, 2], [3, 0, 0]])

    def run():
        cache = jet.KvCache(*(torch.zeros((4, n_kv, 16, dim), dtype=BF16, device="cuda") for _ in range(2)))
        r = [*jet.qk_norm_rope(x, n_q, n_kv, table, pos), *jet.qk_norm_rope(x, n_q, n_kv, table, pos, *gam, 1e-5, cache, slots), cache.k, cache.v]
        r += [*jet.qk_norm_rope_bwd(q, k, x, table, pos, *gam), jet.qk_norm_rope_bwd(q, k, None, table, pos)[0]]
        o, lse = jet.attention_fwd(q, k, v, cu_q=cu, cu_k=cu, causal=False, scale=0.3)
        r += [o, lse, *jet.attention_fwd(q, k, v, cu_q=cu), *jet.attention_bwd(q, k, v, o, lse, do, cu_q=cu, causal=False, scale=0.3)]
        return r + [jet.attention_decode(q[:2], cache, pages, lens), jet.attention_decode(q[:2], cache, pages, lens, 0.3)]

    native = run()
    monkeypatch.setattr(b, "_host", _Declines())
    for i, (s, t) in enumerate(zip(native, run())):
        assert s.dtype == t.dtype and s.shape == t.shape and s.stride() == t.stride() and torch.equal(s, t), i


@pytest.mark.parametrize("native", [True, False])
def test_errors_of_the_library_are_raised(jet, monkeypatch, native):
    from paper_2601_14243_amd import binding as b
    if not native:
        monkeypatch.setattr(b, "_host", _Declines())
    z = lambda *s, dtype=BF16: torch.zeros(s, dtype=dtype, device="cuda")
    calls = [lambda: jet.attention_fwd(z(4, 3, 64), z(4, 2, 64), z(4, 2, 64), cu_q=_i32([0, 4])),              # heads that do not divide
             lambda: jet.attention_fwd(z(4, 4, 96), z(4, 2, 96), z(4, 2, 96), cu_q=_i32([0, 4])),              # channels
             lambda: jet.attention_fwd(z(0, 4, 64), z(4, 2, 64), z(4, 2, 64), cu_q=_i32([0, 0])),              # no rows
             lambda: jet.attention_bwd(z(4, 4, 64), z(4, 2, 64), z(4, 2, 64), z(4, 4, 64), z(4, 4, dtype=torch.float32), z(4, 4, 64), cu_q=_i32([0, 4]), scale=-1.0),
             lambda: jet.qk_norm_rope(z(4, 768), 4, 2, z(9, 96, dtype=torch.float32), _i32([0] * 4)),
             lambda: jet.qk_norm_rope_bwd(z(4, 4, 96), z(4, 2, 96), None, z(9, 96, dtype=torch.float32), _i32([0] * 4)),
             lambda: jet.attention_decode(z(2, 4, 64), jet.KvCache(z(3, 2, 8, 64), z(3, 2, 8, 64)), _i32([[0], [1]]), _i32([1, 1]))]
    for call in calls:
        with pytest.raises(jet.JetError) as e:
            call()
        assert e.value.status in (1, 2, 4)                   # 1: a tensor without rows has no address
    with pytest.raises((TypeError, ValueError)):
        jet.attention_decode(z(2, 4, 64), jet.KvCache(z(3, 2, 16, 128), z(3, 2, 16, 128)), _i32([[0], [1]]), _i32([1, 1]))


def test_long_rows_of_pages_and_many_sequences(jet):
    """A page table far wider than the lengths need, for more sequences than one round of workgroups: chunks that hold no key."""
    lengths = [i * 29 % 300 for i in range(70)]
    cache, x, sc, pages = _paged(jet, lengths, 2, 64, 16, 500, False, seed=120)
    q = _normal(121, (70, 4, 64), 1.5)
    want, tol = ref.decode(q, *x, *sc, pages, lengths, 0.125)
    ref.check(jet.attention_decode(q.cuda(), cache, pages.cuda(), _i32(lengths)), want, tol, "o")


def test_pages_far_into_a_cache(jet):
    """Pages whose first byte lies past 4 GiB and whose elements pass 2^31: written by qk_norm_rope and read as from a small cache."""
    n_q, n_kv, page, dim, T = 16, 8, 128, 128, 300
    n_pages = 2 ** 31 // (n_kv * page * dim) + 40
    far = jet.KvCache(*(torch.empty((n_pages, n_kv, page, dim), dtype=BF16, device="cuda") for _ in range(2)))
    near = jet.KvCache(*(torch.zeros((3, n_kv, page, dim), dtype=BF16, device="cuda") for _ in range(2)))
    x = _normal(140, (T, (n_q + 2 * n_kv) * dim), 1.5).cuda()
    at, pos = torch.arange(T, device="cuda"), torch.arange(T, dtype=torch.int32, device="cuda")
    first = n_pages - 3
    for cache, slots in ((near, at), (far, at + first * page)):
        q, _ = jet.qk_norm_rope(x, n_q, n_kv, _table(dim).cuda(), pos, cache=cache, slots=slots)
    for a, b in ((near.k, far.k), (near.v, far.v)):
        rows = lambda t: t.transpose(1, 2).reshape(3 * page, n_kv, dim)[:T].contiguous().view(torch.int16)
        assert torch.equal(rows(a), rows(b[first:]))
    out = [jet.attention_decode(q[-1:], cache, _i32([[p, p + 1, p + 2]]), _i32([T])) for cache, p in ((near, 0), (far, first))]
    assert out[0].abs().max() > 0 and torch.equal(*(o.view(torch.int16) for o in out))


def test_one_long_sequence_split_over_workgroups(jet):
    """A few thousand rows: several workgroups share the rows of a tile of keys; against float32 on the GPU, products by hand."""
    n, n_q, n_kv, dim = 2500, 8, 2, 64
    q, k, v, do = (_normal(130 + i, (n, h, dim), 1.0).cuda() for i, h in enumerate((n_q, n_kv, n_kv, n_q)))
    cu = _i32([0, n])
    o, lse = jet.attention_fwd(q, k, v, cu_q=cu)
    got = jet.attention_bwd(q, k, v, o, lse, do, cu_q=cu)
    see = ref.visible(n, n, True)
    rows = [0, 1, 127, 128, 1000, 2047, 2499]                # of q: everything; of k and v: sums over all rows
    want = [torch.zeros(x.shape, dtype=torch.float64) for x in (q, k, v)]
    tol = [torch.zeros(x.shape, dtype=torch.float64) for x in (q, k, v)]
    for h in range(n_q):
        g, t = ref.backward(*(x[:, i].cpu().double() for x, i in ((q, h), (k, h // 4), (v, h // 4), (do, h))), dim ** -0.5, see)
        for a, y in ((want, g), (tol, t)):
            a[0][:, h] = y[0]
            a[1][:, h // 4] += y[1]
            a[2][:, h // 4] += y[2]
    for name, a, b_, t in zip(("dq", "dk", "dv"), got, want, tol):
        ref.check(a, b_, t + ref.BF * (b_.abs() + t), name)
    full = ref.forward(q[:, 0].cpu().double(), k[:, 0].cpu().double(), v[:, 0].cpu().double(), dim ** -0.5, see)
    ref.check(o[:, 0][rows], full["o"][rows], full["o_tol"][rows], "o")


@pytest.mark.parametrize("dim,fp8,n_q,n_kv,B,length", [
    (64, False, 4, 2, 3, 700), (128, False, 4, 2, 3, 700), (64, True, 4, 2, 3, 700), (128, True, 8, 8, 3, 700),    # up to 16 chunks of few rows
    (64, False, 4, 2, 2, 2500), (128, True, 4, 2, 2, 2500), (128, False, 4, 4, 1, 9000), (64, False, 16, 8, 80, 1500)])   # the other join
def test_a_bad_page_among_chunks_of_large_scores_gives_nan(jet, dim, fp8, n_q, n_kv, B, length):
    """A sequence of several chunks: the chunk with a page outside the cache is not outweighed by chunks whose scores are far above 104,
    where e^-score is 0 in binary32, whichever of them it is."""
    page = 16
    need = -(-length // page)
    shape = (need + 1, n_kv, page, dim)
    q = torch.full((B, n_q, dim), 4.0, dtype=BF16, device="cuda")
    if fp8:
        k = torch.full(shape, 0x38, dtype=torch.uint8, device="cuda")          # 1.0, times 8
        sc = [torch.full(shape[:3], s, device="cuda") for s in (8.0, 1.0)]
        cache = jet.KvCache(k, k.clone(), *sc)
    else:
        cache = jet.KvCache(torch.full(shape, 8.0, dtype=BF16, device="cuda"), torch.ones(shape, dtype=BF16, device="cuda"))
    assert 4.0 * 8.0 * dim * dim ** -0.5 > 200
    assert jet.jet_attention_decode_workspace(cache._desc_ptr, B, n_q, need) > 0   # several chunks
    pages = torch.arange(need, dtype=torch.int32).repeat(B, 1)
    good = jet.attention_decode(q, cache, pages.cuda(), _i32([length] * B))
    assert (good == 1).all()
    for at in (0, need // 2, need - 1):
        for bad in (-1, need + 1):
            p = pages.clone()
            p[B - 1, at] = bad
            got = jet.attention_decode(q, cache, p.cuda(), _i32([length] * B))
            assert got[B - 1].isnan().all() and (got[:B - 1] == 1).all(), (at, bad)


@pytest.mark.parametrize("native", [True, False])
def test_a_cache_whose_memory_was_replaced_is_refused(jet, monkeypatch, native):
    """The kernels get addresses: a held tensor that lies elsewhere by now is an error, on both host paths, and the cache's tensors cannot be
    exchanged for others."""
    from paper_2601_14243_amd import binding as b
    if not native:
        monkeypatch.setattr(b, "_host", _Declines())
    n_kv, page, dim = 2, 16, 64
    make = lambda: torch.zeros((3, n_kv, page, dim), dtype=BF16, device="cuda")
    q, pages, lens = _normal(150, (1, 4, dim)).cuda(), _i32([[0, 1]]), _i32([20])
    x, table, pos, slots = _normal(151, (1, 8 * dim)).cuda(), _table(dim).cuda(), _i32([3]), torch.tensor([5], device="cuda")
    for i in range(2):
        kv = [make(), make()]
        cache = jet.KvCache(*kv)
        old = kv[i].detach()                                 # keeps the memory
        assert not jet.attention_decode(q, cache, pages, lens).any()
        with pytest.raises(AttributeError):
            setattr(cache, "kv"[i], make())
        kv[i].set_(make())
        with pytest.raises(ValueError):
            jet.attention_decode(q, cache, pages, lens)
        with pytest.raises(ValueError):
            jet.qk_norm_rope(x, 4, n_kv, table, pos, cache=cache, slots=slots)
        assert not kv[i].any() and not old.any()
    like = type("Like", (), {"_where": jet.KvCache(make(), make())._where, "k": make(), "dim": dim})()
    with pytest.raises(TypeError):
        jet.attention_decode(q, like, pages, lens)
