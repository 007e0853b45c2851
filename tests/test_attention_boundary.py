"""Refusals of the attention operators, on the host and before any launch: the C ABI with addresses that are never followed, and the
tensor helpers with CPU tensors that pass for GPU ones."""
import ctypes

import pytest
import torch

from paper_2601_14243_amd import binding as b

A = 0x1000
NULL, SHAPE, ALIGN, ARG = 1, 2, 3, 4
bf, f32, i32, i64, u8 = torch.bfloat16, torch.float32, torch.int32, torch.int64, torch.uint8


def _cache(**kw):
    d = dict(k=A, v=A, k_scale=None, v_scale=None, n_pages=4, n_kv=2, page=16, dim=64)
    d.update(kw)
    return ctypes.pointer(b.KvCacheDesc(*(d[n] for n, _ in b.KvCacheDesc._fields_)))


def _refuses(call, good, wrong):
    """wrong: {position of an argument: [(value, status), ...]}"""
    for i, cases in wrong.items():
        for v, status in cases:
            args = list(good)
            args[i] = v
            assert call(*args) == status, (i, v)


BAD_CACHES = [(dict(k=None), NULL), (dict(v=None), NULL), (dict(k_scale=A), ARG), (dict(v_scale=A), ARG), (dict(page=8), SHAPE), (dict(page=24), SHAPE),
              (dict(page=1 << 17), SHAPE), (dict(dim=96), SHAPE), (dict(n_pages=0), SHAPE), (dict(n_kv=0), SHAPE), (dict(k=A + 8), ALIGN),
              (dict(k_scale=A + 4, v_scale=A), ALIGN)]


def test_qk_norm_rope():
    #        qkv ld  T  n_q n_kv dim table rows pos gq gk eps q  k cache slots stream
    good = [A, 512, 4, 4, 2, 64, A, 100, A, A, A, 1e-6, A, A, None, None, None]
    each = {i: [(None, NULL), (A + 2, ALIGN)] for i in (0, 6, 12, 13)}
    _refuses(b.jet_qk_norm_rope, good, {**each, 1: [(448, SHAPE), (516, SHAPE), ((1 << 24) + 8, SHAPE)], 2: [(0, SHAPE), (1 << 28, SHAPE)],
                                        3: [(0, SHAPE)], 4: [(0, SHAPE)], 5: [(32, SHAPE), (96, SHAPE), (256, SHAPE)], 7: [(0, SHAPE)], 8: [(None, NULL)],
                                        9: [(None, ARG), (A + 8, ALIGN)], 10: [(None, ARG)], 11: [(-1.0, ARG), (float("nan"), ARG), (float("inf"), ARG)],
                                        14: [(_cache(), ARG)], 15: [(A, ARG)]})
    good[14], good[15] = _cache(), A
    _refuses(b.jet_qk_norm_rope, good, {14: [(_cache(**kw), st) for kw, st in BAD_CACHES] + [(_cache(n_kv=4), SHAPE), (_cache(dim=128), SHAPE)]})


def test_qk_norm_rope_bwd():
    #        dq dk qkv ld  T n_q n_kv dim table rows pos gq gk eps dx ld_dx dgq dgk ws stream
    good = [A, A, A, 512, 4, 4, 2, 64, A, 100, A, A, A, 1e-6, A, 384, A, A, A, None]
    each = {i: [(None, NULL), (A + 2, ALIGN)] for i in (0, 1, 2, 8, 14, 16, 17, 18)}
    _refuses(b.jet_qk_norm_rope_bwd, good, {**each, 3: [(448, SHAPE)], 4: [(0, SHAPE)], 7: [(80, SHAPE)], 10: [(None, NULL)], 11: [(None, ARG)],
                                            15: [(376, SHAPE), (388, SHAPE)]})
    plain = list(good)
    plain[11] = plain[12] = None
    assert b.jet_qk_norm_rope_bwd(*plain) == ARG                          # gradients of weights that are not there
    assert b.jet_qk_norm_rope_bwd_workspace(0, 4, 2, 64) == 0 and b.jet_qk_norm_rope_bwd_workspace(1000, 4, 2, 64) > 0


def test_attention_fwd_and_bwd():
    #        q ldq  k ldk  v ldv  cq ck n Tq Tk n_q n_kv dim scale causal o lse stream
    good = [A, 256, A, 128, A, 128, A, A, 2, 8, 8, 4, 2, 64, 0.1, 1, A, A, None]
    shared = {0: [(None, NULL), (A + 2, ALIGN)], 2: [(None, NULL), (A + 2, ALIGN)], 4: [(None, NULL), (A + 2, ALIGN)], 1: [(248, SHAPE), (260, SHAPE)],
              3: [(120, SHAPE)], 5: [((1 << 24) + 8, SHAPE)], 6: [(None, NULL)], 7: [(None, NULL)]}
    sizes = {0: [(0, SHAPE), ((1 << 20) + 1, SHAPE)], 1: [(0, SHAPE), (1 << 28, SHAPE)], 2: [(0, SHAPE), (1 << 29, SHAPE)], 3: [(0, SHAPE), (5, SHAPE)],
             4: [(0, SHAPE), (3, SHAPE)], 5: [(32, SHAPE), (72, SHAPE)], 6: [(0.0, ARG), (-1.0, ARG), (float("nan"), ARG), (float("inf"), ARG)]}
    _refuses(b.jet_attention_fwd, good, {**shared, **{8 + i: c for i, c in sizes.items()}, 16: [(None, NULL), (A + 2, ALIGN)], 17: [(None, NULL), (A + 4, ALIGN)]})
    assert b.jet_attention_fwd(A, 513 * 64 // 8 * 8 + 64, A, 64, A, 64, A, A, 1, 8, 8, 513, 1, 64, 0.1, 1, A, A, None) == SHAPE   # too large a group
    #        ... o lse do cq ck n Tq Tk n_q n_kv dim scale causal dq ld dk ld dv ld ws stream
    back = good[:6] + [A, A, A] + good[6:16] + [A, 256, A, 128, A, 128, A, None]
    wrong = {i: c for i, c in shared.items() if i < 6}
    wrong.update({i: [(None, NULL), (A + 2, ALIGN)] for i in (6, 7, 8, 19, 21, 23, 25)})
    wrong.update({9: [(None, NULL)], 10: [(None, NULL)], 20: [(128, SHAPE)], 22: [(132, SHAPE)], 24: [(64, SHAPE)]})
    wrong.update({11 + i: c for i, c in sizes.items()})
    _refuses(b.jet_attention_bwd, back, wrong)
    assert b.jet_attention_bwd_workspace(1, 0, 8, 4, 2, 64) == 0
    assert b.jet_attention_bwd_workspace(3, 1000, 1000, 4, 2, 64) >= 2 * 4 * 1000 * 4


def test_attention_of_many_keys():
    """The gradients' grid has up to eight workgroups for a tile of keys, the forward pass none of its own for them."""
    #       q ldq  k ldk  v ldv  cq ck n Tq Tk n_q n_kv dim scale causal
    args = [A, 256, A, 128, A, 128, A, A, 2, 8, 1 << 27, 4, 2, 64, 0.1, 1]      # 2^28 keys and heads
    assert b.jet_attention_fwd(*args, A + 2, A, None) == ALIGN            # the sizes are taken, the output is refused
    assert b.jet_attention_bwd(*args[:6], A, A, A, *args[6:], A, 256, A, 128, A, 128, A, None) == SHAPE
    args[9], args[10] = 1 << 28, 8                                        # more query rows than tokens times heads may be
    assert b.jet_attention_fwd(*args, A + 2, A, None) == SHAPE


def test_attention_decode():
    #        q ldq n_q cache pages width lengths B scale o ws stream
    good = [A, 256, 4, _cache(), A, 8, A, 3, 0.1, A, A, None]
    _refuses(b.jet_attention_decode, good, {0: [(None, NULL), (A + 2, ALIGN)], 1: [(248, SHAPE), (260, SHAPE)], 2: [(0, SHAPE), (3, SHAPE)],
                                            3: [(None, NULL)] + [(_cache(**kw), st) for kw, st in BAD_CACHES], 4: [(None, NULL)],
                                            5: [(0, SHAPE), (1 << 28, SHAPE)], 6: [(None, NULL)], 7: [(0, SHAPE), (1 << 28, SHAPE)], 8: [(0.0, ARG), (float("nan"), ARG)],
                                            9: [(None, NULL), (A + 8, ALIGN)], 10: [(A + 4, ALIGN)]})
    assert b.jet_attention_decode_workspace(_cache(), 3, 4, 64) > 0
    good[5], good[10] = 64, None
    assert b.jet_attention_decode(*good) == NULL                          # several chunks without a place for their sums
    assert b.jet_attention_decode_workspace(_cache(), 3, 4, 8) == 0       # one chunk needs none
    assert b.jet_attention_decode_workspace(_cache(page=8), 3, 4, 64) == 0 and b.jet_attention_decode_workspace(None, 3, 4, 64) == 0
    # positions behind the last chunk of a sequence are formed in 32 bits
    assert b.jet_attention_decode_workspace(_cache(page=16), 1, 4, 1 << 26) > 0
    assert b.jet_attention_decode_workspace(_cache(page=16), 1, 4, (1 << 26) + 1) == 0
    good[3], good[5], good[7], good[10] = _cache(page=16), (1 << 27) - 1, 1, A
    assert b.jet_attention_decode(*good) == SHAPE


class _OnGpu(torch.Tensor):
    is_cuda = property(lambda self: True)


def _t(*shape, dtype=bf):
    return torch.zeros(shape, dtype=dtype).as_subclass(_OnGpu)


@pytest.fixture
def no_calls(monkeypatch):
    def called(*a):
        raise AssertionError("a call was made with tensors that do not fit")
    monkeypatch.setattr(b, "_stream", lambda: None)
    for name in ("jet_qk_norm_rope", "jet_qk_norm_rope_bwd", "jet_attention_fwd", "jet_attention_bwd", "jet_attention_decode"):
        monkeypatch.setattr(b, name, called)


def _refused(call, good, wrong):
    for name, values in wrong.items():
        for v in values:
            with pytest.raises((TypeError, ValueError)):
                call(**{**good, name: v})
                pytest.fail(f"{name}: {tuple(v.shape) if isinstance(v, torch.Tensor) else v}")


def test_helpers_refuse_what_does_not_fit(no_calls):
    T, n_q, n_kv, dim = 6, 4, 2, 64
    cpu = torch.zeros
    tb = _t(100, dim, dtype=f32)
    good = dict(qkv=_t(T, 512), n_q=n_q, n_kv=n_kv, table=tb, positions=_t(T, dtype=i32), gamma_q=_t(dim), gamma_k=_t(dim))
    vec = lambda n, dt: [_t(n + 1, dtype=dt), _t(n, dtype=f32 if dt != f32 else bf), _t(n, 1, dtype=dt), _t(2 * n, dtype=dt)[::2], cpu(n, dtype=dt)]
    _refused(b.qk_norm_rope, good, {"qkv": [_t(T, 504), _t(T, 512, dtype=f32), _t(512, T).t(), _t(T, 8, 64), cpu((T, 512), dtype=bf)],
                                    "table": [_t(100, dim), _t(100 * dim, dtype=f32), _t(100, 2 * dim, dtype=f32)[:, :dim]],
                                    "positions": vec(T, i32), "gamma_q": [None, *vec(dim, bf)], "gamma_k": [None, *vec(dim, bf)],
                                    "slots": [_t(T, dtype=i64)]})
    kv = lambda **kw: b.KvCache(_t(4, n_kv, 16, dim), _t(4, n_kv, 16, dim))
    _refused(b.qk_norm_rope, {**good, "cache": kv(), "slots": _t(T, dtype=i64)}, {"slots": [None, *vec(T, i64)], "cache": [None]})
    good = dict(dq=_t(T, n_q, dim), dk=_t(T, n_kv, dim), qkv=_t(T, 512), table=tb, positions=_t(T, dtype=i32), gamma_q=_t(dim), gamma_k=_t(dim))
    head = lambda n: [_t(T, n, dim, dtype=f32), _t(T, n, 128), _t(T, n, 2 * dim)[..., ::2], _t(T, n, 2 * dim)[..., :dim], _t(T + 1, n, dim)]
    _refused(b.qk_norm_rope_bwd, good, {"dq": head(n_q) + [_t(T, n_q + 1, dim)[:, :n_q]], "dk": head(n_kv), "qkv": [_t(T, 448), _t(T + 1, 512)],
                                        "out": [_t(T, 376), _t(T, 384, dtype=f32), _t(T + 1, 384)]})
    cu = _t(3, dtype=i32)
    good = dict(q=_t(T, n_q, dim), k=_t(T, n_kv, dim), v=_t(T, n_kv, dim), cu_q=cu)
    _refused(b.attention_fwd, good, {"q": head(n_q)[:4], "k": head(n_kv)[:4], "v": head(n_kv) + [_t(T, n_kv + 1, dim)],
                                     "cu_q": [_t(3, dtype=i64), _t(3, 1, dtype=i32)], "cu_k": [_t(4, dtype=i32), _t(3, dtype=i64)]})
    good.update(o=_t(T, n_q, dim), lse=_t(n_q, T, dtype=f32), do=_t(T, n_q, dim))
    out = lambda i, v: tuple(v if i == j else t for j, t in enumerate((_t(T, n_q, dim), _t(T, n_kv, dim), _t(T, n_kv, dim))))
    _refused(b.attention_bwd, good, {"o": head(n_q) + [_t(T, n_q + 1, dim)[:, :n_q]], "do": head(n_q), "lse": [_t(T, n_q, dtype=f32), _t(n_q, T)],
                                     "out": [out(i, v) for i, n in enumerate((n_q, n_kv, n_kv)) for v in head(n)]})
    good = dict(q=_t(T, n_q, dim), cache=kv(), pages=_t(T, 5, dtype=i32), lengths=_t(T, dtype=i32))
    _refused(b.attention_decode, good, {"q": [*head(n_q)[:4]], "pages": [_t(T + 1, 5, dtype=i32), _t(T, 5, dtype=i64), _t(T, 10, dtype=i32)[:, ::2]],
                                        "lengths": vec(T, i32)})


def test_cache_refuses_what_does_not_fit():
    k, s = _t(4, 2, 16, 64), _t(4, 2, 16, dtype=f32)
    k8 = _t(4, 2, 16, 64, dtype=u8)
    assert b.KvCache(k, k).page == 16 and b.KvCache(k8, k8, s, s).dim == 64
    for args in ((k, _t(4, 2, 16, 32)), (k8, k8), (k, k, s, s), (k8, k8, s), (k8, k8, s, _t(4, 2, 8, dtype=f32)), (k8, k8, s, _t(4, 2, 16)),
                 (_t(4, 2, 16, 128)[..., :64], k), (torch.zeros((4, 2, 16, 64), dtype=bf), k), (_t(4, 2, 1024), k)):
        with pytest.raises((TypeError, ValueError)):
            b.KvCache(*args)


@pytest.mark.parametrize("fp8", [False, True])
def test_a_cache_whose_memory_was_replaced_is_refused(no_calls, monkeypatch, fp8):
    """The kernels get the addresses that the tensors had when the cache was made."""
    monkeypatch.setattr(b, "_host", type("Declines", (), {"__getattr__": lambda self, name: lambda *a: None})())
    T, dim = 3, 64
    decode = lambda c: b.attention_decode(_t(T, 4, dim), c, _t(T, 5, dtype=i32), _t(T, dtype=i32))
    store = lambda c: b.qk_norm_rope(_t(T, 512), 4, 2, _t(100, dim, dtype=f32), _t(T, dtype=i32), cache=c, slots=_t(T, dtype=i64))
    make = lambda: [_t(4, 2, 16, dim, dtype=u8 if fp8 else bf) for _ in range(2)] + ([_t(4, 2, 16, dtype=f32) for _ in range(2)] if fp8 else [])
    names = ("k", "v", "k_scale", "v_scale")[:len(make())]
    changes = [lambda t: t.set_(torch.zeros_like(t)), lambda t: t.untyped_storage().resize_(0), lambda t: t.untyped_storage().resize_(64),
               lambda t: t.resize_((2,) + tuple(t.shape[1:])), lambda t: t.transpose_(0, 1)]
    for i, name in enumerate(names):
        c = b.KvCache(*make())
        assert getattr(c, name) is not None
        with pytest.raises(AttributeError):
            setattr(c, name, make()[i])
        for change in changes:
            ts = make()
            c = b.KvCache(*ts)
            change(ts[i])
            for call in (decode, store):
                with pytest.raises(ValueError, match=f"memory of {name} "):
                    call(c)
    for name in ("n_pages", "n_kv", "page", "dim"):
        with pytest.raises(AttributeError):
            setattr(c, name, 8)


def test_what_only_looks_like_a_cache_is_refused(no_calls, monkeypatch):
    monkeypatch.setattr(b, "_host", type("Declines", (), {"__getattr__": lambda self, name: lambda *a: None})())
    c = b.KvCache(_t(4, 2, 16, 64), _t(4, 2, 16, 64))
    like = type("Like", (), dict(k=c.k, v=c.v, dim=64, _desc_ptr=c._desc_ptr, _where=c._where))()
    for call in (lambda x: b.attention_decode(_t(3, 4, 64), x, _t(3, 5, dtype=i32), _t(3, dtype=i32)),
                 lambda x: b.qk_norm_rope(_t(3, 512), 4, 2, _t(100, 64, dtype=f32), _t(3, dtype=i32), cache=x, slots=_t(3, dtype=i64))):
        with pytest.raises(TypeError, match="KvCache"):
            call(like)


def test_native_marshalling_declines_all_but_the_plain_form():
    h = b._native()
    q, cu = torch.zeros((4, 2, 64), dtype=bf), torch.zeros(2, dtype=i32)
    assert h.qk_norm_rope(torch.zeros((4, 512), dtype=bf), 4, 2, torch.zeros((9, 64)), torch.zeros(4, dtype=i32), None, None, 1e-6, None, None) is None
    assert h.qk_norm_rope_bwd(q, q, None, torch.zeros((9, 64)), torch.zeros(4, dtype=i32), None, None, 1e-6) is None
    assert h.attention_fwd(q, q, q, cu, None, True, None) is None
    assert h.attention_bwd(q, q, q, q, torch.zeros((2, 4)), q, cu, None, True, None) is None
    assert h.attention_decode(q, None, torch.zeros((4, 2), dtype=i32), torch.zeros(4, dtype=i32), None) is None
    with pytest.raises(TypeError):
        h.attention_fwd(q, q, q)
