"""Refusals of the embedding, layer norm and clipping operators, on the host and before any launch: the C ABI with addresses that are never
followed, and the tensor helpers with CPU tensors that pass for GPU ones."""
import ctypes
import math

import pytest
import torch

from paper_2601_14243_amd import binding as b

A = 0x1000
NULL, SHAPE, ALIGN, ARG = 1, 2, 3, 4
bf, f32, f16, i32, i64, u8 = torch.bfloat16, torch.float32, torch.float16, torch.int32, torch.int64, torch.uint8
nan, inf = float("nan"), float("inf")


def _refuses(call, good, wrong):
    """wrong: {position of an argument: [(value, status), ...]}"""
    for i, cases in wrong.items():
        for v, status in cases:
            args = list(good)
            args[i] = v
            assert call(*args) == status, (i, v)


SIZES = {2: [(0, SHAPE), (-1, SHAPE), ((1 << 22) + 1, SHAPE)]}
EPS = [(-1.0, ARG), (nan, ARG), (inf, ARG)]


def test_embedding():
    #        ids type T  w  type V    H   first scale y stream
    good = [A, 0, 4, A, 1, 100, 64, 0, 1.0, A, None]
    each = {i: [(None, NULL), (A + 4, ALIGN)] for i in (0, 3, 9)}
    _refuses(b.jet_embedding_fwd, good, {**each, **SIZES, 1: [(2, ARG), (-1, ARG)], 4: [(2, ARG)], 5: [(0, SHAPE), (1 << 31, SHAPE)],
                                         6: [(0, SHAPE), (4, SHAPE), (60, SHAPE), ((1 << 20) + 8, SHAPE)], 7: [((1 << 62) + 1, SHAPE), (-(1 << 62) - 1, SHAPE)],
                                         8: [(nan, ARG), (inf, ARG)]})
    #        ids type T  dy V    H   first scale dw type add ws stream
    good = [A, 0, 4000, A, 100, 64, 0, 1.0, A, 1, 0, A, None]
    each = {i: [(None, NULL), (A + 8, ALIGN)] for i in (0, 3, 8, 11)}
    _refuses(b.jet_embedding_bwd, good, {**each, **SIZES, 1: [(3, ARG)], 4: [(0, SHAPE), (1 << 31, SHAPE)], 5: [(0, SHAPE), (100, SHAPE)],
                                         6: [((1 << 62) + 1, SHAPE)], 7: [(nan, ARG), (-inf, ARG)], 9: [(2, ARG)]})
    good[2], good[5] = 1 << 18, 1 << 19                                  # tokens times columns
    assert b.jet_embedding_bwd(*good) == SHAPE
    assert b.jet_embedding_bwd_workspace(0, 64) == 0 and b.jet_embedding_bwd_workspace(1, 64) == 0 and b.jet_embedding_bwd_workspace(4000, 64) > 0
    assert b.jet_embedding_bwd_workspace((1 << 22) + 1, 64) == 0


def test_layernorm():
    #        x  res gamma beta eps M  K   sum  y  q  s  stream
    good = [A, A, A, A, 1e-5, 4, 256, A, A, None, None, None]
    each = {i: [(None, NULL), (A + 8, ALIGN)] for i in (0, 2)}
    _refuses(b.jet_layernorm_fwd, good, {**each, 1: [(None, ARG), (A + 2, ALIGN)], 3: [(A + 2, ALIGN)], 4: EPS,
                                         5: [(0, SHAPE), ((1 << 23) + 1, SHAPE)], 6: [(0, SHAPE), (252, SHAPE), (32776, SHAPE)], 7: [(None, ARG), (A + 2, ALIGN)],
                                         8: [(None, ARG), (A + 2, ALIGN)], 9: [(A, ARG)], 10: [(A, NULL)]})
    good[8:11] = [None, A, A]
    _refuses(b.jet_layernorm_fwd, good, {6: [(264, SHAPE)], 8: [(A, ARG)], 9: [(None, ARG), (A + 8, ALIGN)], 10: [(None, NULL), (A + 4, ALIGN)]})
    for M, K in ((1 << 19) + 1, 32768), ((1 << 21) + 1, 8192), (1 << 23, 4096), (1 << 23, 2176):      # more values than a launch has threads for
        good[5], good[6] = M, K
        assert b.jet_layernorm_fwd(*good) == SHAPE
        assert b.jet_norm_bwd(b.JET_NORM_LAYER, A, A, A, A, 1e-5, M, K, A, A, A, A, None) == SHAPE and b.jet_norm_bwd_workspace(0, M, K) == 0


def test_norm_bwd():
    #        kind dy x gamma dres eps M K dx dgamma dbeta ws stream
    good = [b.JET_NORM_LAYER, A, A, A, A, 1e-5, 4, 256, A, A, A, A, None]
    each = {i: [(None, NULL), (A + 8, ALIGN)] for i in (1, 2, 3, 8, 9, 10, 11)}
    wrong = {**each, 0: [(2, ARG), (-1, ARG)], 4: [(A + 2, ALIGN)], 5: EPS, 6: [(0, SHAPE)], 7: [(0, SHAPE), (12, SHAPE), (32776, SHAPE)]}
    _refuses(b.jet_norm_bwd, good, wrong)
    good[0], good[10] = b.JET_NORM_RMS, None
    del wrong[0]
    _refuses(b.jet_norm_bwd, good, {**wrong, 10: [(A, ARG)]})
    assert b.jet_norm_bwd_workspace(0, 0, 256) == 0 and b.jet_norm_bwd_workspace(0, 4, 252) == 0
    assert b.jet_norm_bwd_workspace(0, 1000, 256) == 2 * b.jet_norm_bwd_workspace(1, 1000, 256) > 0


def _descs(*t):
    return (b.TensorDesc * len(t))(*[b.TensorDesc(*x) for x in t])


def test_clipping():
    one = _descs((A, 100, 0), (A + 4096, 7, 1), (None, 0, 0))
    bad = [(_descs((None, 3, 0)), NULL), (_descs((A, -1, 0)), SHAPE), (_descs((A, (1 << 40) + 1, 0)), SHAPE), (_descs((A, 3, 2)), ARG), (_descs((A + 8, 3, 0)), ALIGN)]
    good = [one, 3, A, A, None]
    _refuses(b.jet_grad_norm, good, {0: [(None, NULL)], 1: [(0, SHAPE), (-1, SHAPE), ((1 << 16) + 1, SHAPE)], 2: [(None, NULL), (A + 4, ALIGN)],
                                     3: [(None, NULL), (A + 8, ALIGN)]})
    for t, status in bad:
        assert b.jet_grad_norm(t, 1, A, A, None) == status
        assert b.jet_clip_grads(t, None, 1, 1.0, None, A, A, None) == status
    #       tensors out n max given norm ws stream
    good = [one, None, 3, 1.0, None, A, A, None]
    _refuses(b.jet_clip_grads, good, {0: [(None, NULL)], 2: [(0, SHAPE)], 3: [(-1.0, ARG), (nan, ARG)], 4: [(A + 4, ALIGN)], 5: [(A + 4, ALIGN)],
                                      6: [(None, NULL), (A + 8, ALIGN)]})
    far, norm = 1 << 30, 1 << 40
    fits = _descs((far, 100, 0), (far + 4096, 7, 1), (None, 0, 0))
    for out, status in ((_descs((far, 99, 0), (far + 4096, 7, 1), (None, 0, 0)), SHAPE), (_descs((far, 100, 1), (far + 4096, 7, 1), (None, 0, 0)), SHAPE)):
        assert b.jet_clip_grads(one, out, 3, 1.0, None, A, A, None) == status
    # memory that is written and belongs to two tensors
    for t, out in ((_descs((A, 100, 0), (A, 100, 0)), None), (_descs((A, 100, 0), (A + 192, 5, 1)), None), (_descs((A, 1000, 0), (A + 4000, 5, 1), (A + 16, 1, 0)), None),
                   (one, one), (one, _descs((far, 100, 0), (far + 192, 7, 1), (None, 0, 0))), (one, _descs((A + 192, 100, 0), (far, 7, 1), (None, 0, 0))),
                   (_descs(*[(A + 4096 * i, 100, 0) for i in range(300)], (A + 4096 * 77, 1, 1)), None)):
        n = len(t)
        assert b.jet_clip_grads(t, out, n, 1.0, None, norm, A, None) == ARG
    # the norm among the tensors
    for out in (None, fits):
        assert b.jet_clip_grads(one, out, 3, 1.0, None, A + 192, A, None) == ARG
    assert b.jet_clip_grads(one, None, 3, 1.0, A + 192, None, None, None) == ARG
    assert b.jet_clip_grads(one, fits, 3, 1.0, far + 4096 + 16, None, None, None) == ARG
    assert b.jet_clip_grads(one, fits, 3, 1.0, norm, norm, None, None) == ARG
    assert b.jet_grad_norm_workspace(0) == 0 and b.jet_grad_norm_workspace((1 << 16) + 1) == 0 and b.jet_grad_norm_workspace(1) > 0


class _OnGpu(torch.Tensor):
    is_cuda = property(lambda self: True)


def _t(*shape, dtype=bf):
    return torch.zeros(shape, dtype=dtype).as_subclass(_OnGpu)


@pytest.fixture
def no_calls(monkeypatch):
    def called(*a):
        raise AssertionError("a call was made with tensors that do not fit")
    monkeypatch.setattr(b, "_stream", lambda: None)
    for name in ("jet_embedding_fwd", "jet_embedding_bwd", "jet_layernorm_fwd", "jet_norm_bwd", "jet_grad_norm", "jet_clip_grads"):
        monkeypatch.setattr(b, name, called)


def _refused(call, good, wrong):
    for name, values in wrong.items():
        for v in values:
            with pytest.raises((TypeError, ValueError)):
                call(**{**good, name: v})
                pytest.fail(f"{name}: {tuple(v.shape) if isinstance(v, torch.Tensor) else v}")


def test_helpers_refuse_what_does_not_fit(no_calls):
    T, H, V = 6, 64, 9
    cpu = torch.zeros
    ids = [_t(T, dtype=f32), _t(T, 1, dtype=i64), _t(2 * T, dtype=i64)[::2], cpu(T, dtype=i64), _t(T, dtype=torch.int16)]
    mat = lambda m, n, dt=bf: [_t(m, n + 8, dtype=dt), _t(m, 2 * n, dtype=dt)[:, :n], _t(n, m, dtype=dt).t(), _t(m, n, dtype=f16), cpu((m, n), dtype=dt), _t(m * n, dtype=dt)]
    _refused(b.embedding_fwd, dict(ids=_t(T, dtype=i64), w=_t(V, H)), {"ids": ids, "w": mat(V, H)[1:], "out": mat(T, H) + [_t(T, H, dtype=f32), _t(T + 1, H)],
                                                                       "first": [1 << 63, -(1 << 63)]})
    good = dict(ids=_t(T, dtype=i32), dy=_t(T, H), rows=V)
    _refused(b.embedding_bwd, good, {"ids": ids + [_t(T + 1, dtype=i64)], "dy": mat(T, H)[1:] + [_t(T, H, dtype=f32), _t(T + 1, H)], "dtype": [f16, torch.float64, i32],
                                     "out": mat(V, H) + [_t(V + 1, H)], "accumulate": [True], "first": [1 << 63], "rows": [0, -1, 1 << 31]})
    vec = lambda n: [_t(n + 1), _t(n, dtype=f32), _t(n, 1), _t(2 * n)[::2], cpu(n, dtype=bf)]
    good = dict(x=_t(T, H), gamma=_t(H), beta=_t(H), eps=1e-5)
    _refused(b.layernorm_fwd, good, {"x": mat(T, H) + [_t(T, H, dtype=f32)], "gamma": vec(H), "beta": vec(H), "residual": mat(T, H) + [_t(T + 1, H), _t(T, H, dtype=f32)]})
    for f in (b.layernorm_bwd, b.rmsnorm_bwd):
        good = dict(dy=_t(T, H), x=_t(T, H), gamma=_t(H), eps=1e-5)
        _refused(f, good, {"dy": mat(T, H) + [_t(T + 1, H)], "x": mat(T, H) + [_t(T, H, dtype=f32)], "gamma": vec(H), "dres": mat(T, H) + [_t(1, H)]})
    lists = [[], _t(3), None, [_t(3), cpu(3)], [_t(3, dtype=f16)], [_t(4, 6)[:, :3]], [_t(3), 1.0], {"a": _t(3)}]
    _refused(b.grad_norm, {}, {"grads": lists})
    good = dict(grads=[_t(3), _t(2, 2, dtype=f32)], max_norm=1.0)
    _refused(b.clip_grads, good, {"grads": lists, "out": lists[1:2] + lists[3:] + [[_t(3)], [_t(4), _t(2, 2, dtype=f32)], [_t(3), _t(2, 2)], [_t(3), _t(4, dtype=f32)]],
                                  "norm": [_t(2, dtype=f32), _t(1), cpu(1)]})


def test_native_marshalling_declines_all_but_the_plain_form():
    h = b._native()
    x, ids = torch.zeros((4, 64), dtype=bf), torch.zeros(4, dtype=i64)
    assert h.embedding_fwd(ids, x, 1.0, 0, None) is None
    assert h.embedding_bwd(ids, x, 9, 1.0, 0, True, None, False) is None
    assert h.layernorm_fwd(x, x[0], None, 1e-5, None, False) is None
    assert h.norm_bwd(0, x, x, x[0], 1e-5, None) is None
    for grads in ([x], (x,), [], [1], "x", None):
        assert h.clip_grads(grads, 1.0, None, None) is None and h.clip_grads(grads, None, None, None) is None
    with pytest.raises(TypeError):
        h.norm_bwd(0, x, x)
    assert all(getattr(b._PythonMarshalling, n)() is None for n in ("embedding_fwd", "embedding_bwd", "layernorm_fwd", "norm_bwd", "clip_grads"))


def test_operands_on_another_device_than_the_current_one_are_refused(monkeypatch):
    """Streams, allocations and launches go by the current device."""
    class Elsewhere(_OnGpu):
        device = property(lambda self: torch.device("cuda", 1))
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    monkeypatch.setattr(torch, "empty", lambda *a, **k: _t(4, 64).as_subclass(Elsewhere))
    monkeypatch.setattr(torch, "empty_like", lambda t: t)
    e = lambda *s, dtype=bf: torch.zeros(s, dtype=dtype).as_subclass(Elsewhere)
    for call in (lambda: b.embedding_fwd(e(4, dtype=i64), e(9, 64)), lambda: b.layernorm_fwd(e(4, 64), e(64), None, 1e-5),
                 lambda: b.layernorm_bwd(e(4, 64), e(4, 64), e(64), 1e-5), lambda: b.grad_norm([e(4)]), lambda: b.clip_grads([e(4)], 1.0),
                 lambda: b.embedding_bwd(e(4, dtype=i64), e(4, 64), 4, dtype=bf)):
        with pytest.raises(ValueError, match="current device"):
            call()


def test_clipping_to_no_norm_is_refused(no_calls):
    good = dict(grads=[_t(3), _t(2, 2, dtype=f32)], max_norm=1.0)
    _refused(b.clip_grads, good, {"max_norm": [None, [1.0], "one"]})
    _refused(b.clip_grads, {**good, "out": [_t(3), _t(2, 2, dtype=f32)], "norm": _t(1, dtype=f32)}, {"max_norm": [None]})
