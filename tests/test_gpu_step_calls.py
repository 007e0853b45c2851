"""Calls of the embedding, norm and clipping operators that their documentation allows and that are easily answered wrongly, each
through the native and the Python path where the two might differ."""
import math

import pytest
import torch

import step_ref as ref
from test_gpu_step import _f32, _gen, _grads, _normal, _same, bf, f32, f64, i32, i64, jet  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.fixture(params=["native", "python"])
def path(request, jet, monkeypatch):  # noqa: F811
    """The helpers by way of the extension, or with all calls declined by it."""
    from paper_2601_14243_amd import binding
    if request.param == "python":
        monkeypatch.setattr(binding, "_host", type("Declines", (), {"__getattr__": lambda self, name: lambda *a: None})())
    else:
        assert binding._native() is not binding._PythonMarshalling
    return request.param


def test_clipping_of_tensors_that_share_memory_until_they_are_written(jet, path):
    """A lazy clone is a tensor of its own: it is scaled or written, the one that it was made of stays."""
    g = _gen(1)
    grads = [_normal(g, (n,), 1.0, t) for n, t in ((3000, f32), (20000, bf), (5, bf))]
    before = [t.clone() for t in grads]
    want, tol = ref.clipped(grads, 1.0)
    lazy = [torch._lazy_clone(t) for t in grads]
    assert all(torch._C._data_address(a) == torch._C._data_address(b) for a, b in zip(lazy, grads))
    norm = jet.clip_grads(lazy, 1.0)                                     # in place
    assert all(_same(a, b) for a, b in zip(grads, before))
    for a, b, t in zip(lazy, want, tol):
        ref.check(a, b, t, "in place")
    to = [torch._lazy_clone(t) for t in grads]
    assert _same(jet.clip_grads(grads, 1.0, out=to), norm)               # into clones of what is read
    assert all(_same(a, b) for a, b in zip(grads, before)) and all(_same(a, b) for a, b in zip(to, lazy))
    other = [torch.full_like(t, 3.0) for t in grads]
    to = [torch._lazy_clone(t) for t in other]
    jet.clip_grads([torch._lazy_clone(t) for t in grads], 1.0, out=to)   # into clones of others, from clones
    assert all(bool((t == 3.0).all()) for t in other) and all(_same(a, b) for a, b in zip(to, lazy))
    assert all(_same(a, b) for a, b in zip(grads, before))
    both = [grads[0], torch._lazy_clone(grads[0])]                       # one beside its clone
    jet.clip_grads(both, 1.0)
    assert _same(both[0], both[1]) and torch._C._data_address(both[0]) != torch._C._data_address(both[1])
    ref.check(both[1], *(v[0] for v in ref.clipped([before[0], before[0]], 1.0)), "beside its clone")
    same = torch._lazy_clone(grads[1])
    with pytest.raises(jet.JetError, match="status 4"):                  # overlaps itself, shared or not
        jet.clip_grads([same], 1.0, out=[same])
    read = torch._lazy_clone(grads[1])
    assert _same(jet.grad_norm([read]), jet.grad_norm([grads[1]]))       # only read: still shared
    assert path == "python" or torch._C._data_address(read) == torch._C._data_address(grads[1])


def test_clipping_without_a_norm_to_clip_to_is_refused(jet, path):
    """Not answered by the norm alone, with the outputs unwritten."""
    grads = _grads(_gen(2), [100, 3000])
    before, to = [t.clone() for t in grads], [torch.full_like(t, 9.0) for t in grads]
    for kw in (dict(), dict(out=to), dict(norm=torch.tensor(2.0, device="cuda")), dict(norm=torch.tensor(2.0, device="cuda"), out=to)):
        with pytest.raises(TypeError):
            jet.clip_grads(grads, None, **kw)
    assert all(_same(a, b) for a, b in zip(grads, before)) and all(bool((t == 9.0).all()) for t in to)
    assert _same(jet.grad_norm(grads), jet.clip_grads(grads, math.inf))  # infinity: the norm, and nothing is scaled


def test_a_first_id_out_of_range_is_the_same_error_on_both_paths(jet, path):
    ids, w = torch.zeros(4, dtype=i64, device="cuda"), torch.ones((9, 64), dtype=bf, device="cuda")
    dy = torch.ones((4, 64), dtype=bf, device="cuda")
    for first in ((1 << 62) + 1, -(1 << 62) - 1, (1 << 63) - 1, -(1 << 63), 1 << 63, 1 << 80):
        for call in (lambda: jet.embedding_fwd(ids, w, first=first), lambda: jet.embedding_bwd(ids, dy, 9, first=first)):
            with pytest.raises(ValueError, match="first"):
                call()
    for first in (1 << 62, -(1 << 62)):                                  # the last ones that are taken: no token has a row
        assert not jet.embedding_fwd(ids, w, first=first).any() and not jet.embedding_bwd(ids, dy, 9, first=first).any()


@pytest.mark.parametrize("value,max_norm", [(2e36, 1e-3), (2e36, 1e-6), (1e36, 1e-8), (2e36, 1e-20), (1e36, 1e-36), (1e36, 1e-40), (1.0, 1e-37), (1e-3, 1e-40),
                                            (1e20, 1e-17), (1.0, 0.0)])
def test_a_factor_below_the_normal_numbers_of_binary32(jet, value, max_norm):
    """Gradients that exploded, or hardly any norm to clip to: max_norm / norm keeps its bits, and what it scales is not zero."""
    g = _gen(8)
    grads = [(_normal(g, (n,), 1.0, f32) * value).to(t) for n, t in ((300, f32), (8192, bf), (9001, bf), (8195, f32), (1, bf))]
    max32 = _f32(max_norm)
    total = ref.norm(grads)
    assert math.isfinite(_f32(total)) and max32 / total < 2.0 ** -120
    want, tol = ref.clipped(grads, max32)
    to = [torch.full_like(t, 9.0) for t in grads]
    norm = jet.clip_grads(grads, max_norm, out=to)
    mine, beside = [t.clone() for t in grads], [t.clone() for t in grads]
    assert _same(jet.clip_grads(mine, max_norm), norm)
    jet.clip_grads(beside, max_norm, norm=norm)
    beside_want, beside_tol = ref.clipped(grads, max32, norm.item())
    for a, b, w, t, c, cw, ct in zip(to, mine, want, tol, beside, beside_want, beside_tol):
        ref.check(a, w, t, "out")
        assert _same(a, b)
        ref.check(c, cw, ct, "by the norm that is given")
    if max32 >= 1e-30:                                                   # (smaller ones lose elements below 2^-149)
        assert abs(ref.norm(to) - max32) <= max32 * (ref.BF + 2 * ref.F) * 1.01


# many tensors, whose norm has a launch of its own: little more than one launch's partial sums, nothing in some tensors, the most there may be
MANY_TENSORS = [[10] * 2100, [(i * 37) % 30000 for i in range(1300)], [i % 5 for i in range(1 << 16)]]
LARGE, FEW = [50_000_000, 70_000_001], [3000, 20000, 5]


@pytest.mark.parametrize("sizes", MANY_TENSORS, ids=len)
def test_clipping_of_many_tensors(jet, sizes):
    g = _gen(len(sizes))
    flat = {t: _normal(g, (sum(-(-n // 8) * 8 for n in sizes),), 1.0, t) for t in (bf, f32)}

    def views(flat):
        at, out = 0, []
        for i, n in enumerate(sizes):
            out.append(flat[bf if i % 3 else f32][at:at + n])
            at += -(-n // 8) * 8
        return out

    grads = views(flat)
    joined = [torch.cat([t for t in grads if t.dtype == d]) for d in (bf, f32)]
    want = ref.norm(joined)
    norm = jet.grad_norm(grads)
    assert abs(norm.item() - want) <= want * ref.F * 1.01
    for max_norm in (0.4 * want, 2.0 * want):
        expect, tol = ref.clipped(joined, _f32(max_norm))
        mine, to = views({d: t.clone() for d, t in flat.items()}), views({d: torch.full_like(t, 9.0) for d, t in flat.items()})
        for kw, result in ((dict(), mine), (dict(out=to), to)):
            assert _same(jet.clip_grads(mine if result is mine else grads, max_norm, **kw), norm)
            for d, e, t in zip((bf, f32), expect, tol):
                ref.check(torch.cat([v for v in result if v.dtype == d]), e, t, "scaled")


def test_every_form_of_clipping_replayed_from_a_graph(jet):
    """In place and to new tensors, small and large, many tensors, by a norm that is given: the norm in launches of its own and not; other inputs in each
    replay, which reach the limit or do not."""
    g = _gen(60)
    lists = [_grads(g, s) for s in (FEW, LARGE, MANY_TENSORS[1])]
    limit = [math.sqrt(sum(t.numel() for t in ts)) for ts in lists]
    given = torch.tensor(3.0, device="cuda")

    def calls(lists):
        norms = []
        for ts, most in zip(lists, limit):
            to, by = [torch.empty_like(t) for t in ts], [torch.empty_like(t) for t in ts]
            norms += [jet.grad_norm(ts), jet.clip_grads(ts, most, out=to), jet.clip_grads(ts, 2.0, norm=given, out=by), *to, *by]
            norms.append(jet.clip_grads(ts, most))                       # in place
            norms += ts
        return norms

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        calls(lists)
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = calls(lists)
    for rep in range(4):
        given.fill_(1.0 + 2 * (rep % 2))
        for i, ts in enumerate(lists):
            for t in ts:
                t.copy_(_normal(g, t.shape, 3.0 if (rep + i) % 2 else 0.3, t.dtype))
        eager = [[t.clone() for t in ts] for ts in lists]
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in out]
        want = calls(eager)
        assert len(got) == len(want) and all(_same(a, b) for a, b in zip(got, want)), rep
        for ts, most in zip(eager, limit):                               # scaled, or as they were
            assert all(bool(t.isfinite().all()) for t in ts) and jet.grad_norm(ts).item() <= most * 1.01


@pytest.mark.parametrize("M,K", [(5, 64), (9, 1000), (1100, 1000), (3, 4096), (1100, 4096), (7, 8200), (5, 32768)])
@pytest.mark.parametrize("power", [61, -54])
def test_norms_at_the_ends_of_their_range(jet, M, K, power):
    """Variances of 2^122 and 2^-108, without eps, in rows beside ordinary ones."""
    g = _gen(M + K)
    x, gamma, beta, dy = _normal(g, (M, K)), 1 + _normal(g, (K,), 0.2), _normal(g, (K,), 0.1), _normal(g, (M, K), 1e-3)
    x[::2] *= 2.0 ** power
    ref.check(jet.layernorm_fwd(x, gamma, beta, 0.0)["y"], *ref.layer_norm(x, gamma, beta, 0.0), "y")
    for f, layer in ((jet.layernorm_bwd, True), (jet.rmsnorm_bwd, False)):
        want, tol = ref.norm_backward(dy, x, gamma, 0.0, None, layer)
        for a, b, t, name in zip(f(dy, x, gamma, 0.0), want, tol, ("dx", "dgamma", "dbeta")):
            ref.check(a, b, t, name)
