// Native marshalling for binding.py: the checks, output allocations and C-ABI calls of the tensor helpers in
// one Python call each.  A small layer is bound by what the host does per launch: through ctypes and a dozen tensor
// attributes quant_act took 11.1 us, a GEMM call 11.6, quant_weight with its copy 14.8; here 5.3, 4.3 and 6.9.
//
// Every function returns None when a call is not of the plain form (exact torch tensors on one GPU, of the expected
// dtype, layout and shapes, outputs included; `out` absent or complete): binding.py then takes its Python path, which words
// the error or handles the unusual form.  Only calls that that path would accept are answered here, with the same results.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <ATen/core/Tensor.h>
#include <ATen/hip/EmptyTensor.h>
#include <ATen/ops/empty.h>
#include <ATen/PythonTorchFunctionTLS.h>
#include <c10/hip/HIPCachingAllocator.h>
#include <c10/hip/HIPFunctions.h>
#include <c10/hip/HIPStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include <algorithm>
#include <cmath>

#include "../../include/jet.h"

namespace {

PyObject* g_error = nullptr;   // binding.JetError
PyObject* g_oom = nullptr;     // torch.OutOfMemoryError
PyObject* g_cache = nullptr;   // binding.KvCache

constexpr int64_t kGroup = 128;

// nullptr unless obj is a torch.Tensor or Parameter itself on the GPU with dtype
const at::Tensor* plain(PyObject* obj, at::ScalarType dtype) {
    if (!THPVariable_CheckExact(obj)) return nullptr;
    const at::Tensor& t = THPVariable_Unpack(obj);
    return (t.is_cuda() && t.scalar_type() == dtype) ? &t : nullptr;
}
const at::Tensor* plain2d(PyObject* obj, at::ScalarType dtype) {
    const at::Tensor* t = plain(obj, dtype);
    return (t && t->dim() == 2 && t->is_contiguous()) ? t : nullptr;
}
// t may hold [rows, cols] densely from its start (binding.py's _need_rows): on like's device, contiguous, of the element
// size, with room, and with rows of `cols` unless it is flat
enum Kind { kCodes, kScales };
bool holds(const at::Tensor& t, Kind kind, int64_t rows, int64_t cols, const at::Tensor& like) {
    cols = std::max<int64_t>(cols, 1);
    return t.is_cuda() && t.device() == like.device() && t.is_contiguous() &&
           (kind == kCodes ? t.element_size() == 1 : t.scalar_type() == at::kFloat) && t.numel() >= rows * cols &&
           (t.dim() == 1 || (t.dim() > 1 && t.size(-1) == cols));
}
bool modes_active() { return at::impl::torch_function_mode_enabled(); }
void* stream() { return c10::hip::getCurrentHIPStream().stream(); }
at::Tensor make(int64_t rows, int64_t cols, at::ScalarType dtype, const at::Tensor& like) {
    return at::empty({rows, cols}, at::TensorOptions().dtype(dtype).device(like.device()));
}
template <class T = uint8_t>
const T* in(const at::Tensor& t) { return static_cast<const T*>(t.const_data_ptr()); }
template <class T = uint8_t>
T* outp(const at::Tensor& t) { return static_cast<T*>(t.data_ptr()); }

// nullptr with JetError set when st is an error, else the new reference `result`
PyObject* finish(jet_status st, const char* where, PyObject* result) {
    if (st == JET_OK) return result;
    Py_XDECREF(result);
    PyObject* e = PyObject_CallFunction(g_error, "is", (int)st, where);
    if (e) {
        PyErr_SetObject(g_error, e);
        Py_DECREF(e);
    }
    return nullptr;
}
// C++ exceptions of the allocator and of torch do not cross into Python as such
template <class F>
PyObject* guarded(F&& f) {
    try {
        return f();
    } catch (const python_error&) {
        return nullptr;       // already set
    } catch (const c10::OutOfMemoryError& e) {
        PyErr_SetString(g_oom, e.what_without_backtrace());
    } catch (const c10::Error& e) {
        PyErr_SetString(PyExc_RuntimeError, e.what_without_backtrace());
    } catch (const std::exception& e) {
        PyErr_SetString(PyExc_RuntimeError, e.what());
    }
    return nullptr;
}
bool set_item(PyObject* d, const char* key, const at::Tensor& t) {
    PyObject* o = THPVariable_Wrap(t);
    if (!o) return false;
    const int r = PyDict_SetItemString(d, key, o);
    Py_DECREF(o);
    return r == 0;
}
// a pair of result tensors of a quantizer: new ones, or those of the caller's dict
struct Pair {
    at::Tensor q, s;
};
// codes [rows, cols] with scales [rows, cols / 128]; false: not of the plain form
bool take_pair(PyObject* out, const char* qk, const char* sk, int64_t rows, int64_t cols, const at::Tensor& like, Pair& p) {
    PyObject *q = PyDict_GetItemString(out, qk), *s = PyDict_GetItemString(out, sk);
    if (!q || !s || !THPVariable_CheckExact(q) || !THPVariable_CheckExact(s)) return false;
    p.q = THPVariable_Unpack(q);
    p.s = THPVariable_Unpack(s);
    return holds(p.q, kCodes, rows, cols, like) && holds(p.s, kScales, rows, cols / kGroup, like);
}
PyObject* dict_of(const Pair* row, const Pair* col) {
    PyObject* d = PyDict_New();
    if (!d) return nullptr;
    if ((row && !(set_item(d, "q_row", row->q) && set_item(d, "s_row", row->s))) ||
        (col && !(set_item(d, "q_colT", col->q) && set_item(d, "s_colT", col->s)))) {
        Py_DECREF(d);
        return nullptr;
    }
    return d;
}
PyObject* same_or(PyObject* out, const Pair* row, const Pair* col) {
    if (out == Py_None) return dict_of(row, col);
    Py_INCREF(out);
    return out;
}
bool args(Py_ssize_t have, Py_ssize_t want) {
    if (have == want) return true;
    PyErr_SetString(PyExc_TypeError, "wrong number of arguments");
    return false;
}

// quant_act(x, x_scales | None, row, col, out | None)
PyObject* quant_act(PyObject*, PyObject* const* a, Py_ssize_t n) {
    if (!args(n, 5)) return nullptr;
    return guarded([&]() -> PyObject* {
        const bool fp8 = a[1] != Py_None;
        const int row = PyObject_IsTrue(a[2]), col = PyObject_IsTrue(a[3]);
        if (row < 0 || col < 0) return nullptr;
        PyObject* out = a[4];
        const at::Tensor* x = plain2d(a[0], fp8 ? at::kByte : at::kBFloat16);
        const at::Tensor* xs_t = fp8 ? plain(a[1], at::kFloat) : nullptr;
        if (!x || (fp8 && !xs_t) || (out != Py_None && !PyDict_CheckExact(out)) || modes_active()) Py_RETURN_NONE;
        const int64_t M = x->size(0), K = x->size(1);
        if (fp8 && !holds(*xs_t, kScales, M, K / kGroup, *x)) Py_RETURN_NONE;
        Pair r, c;
        if (out != Py_None) {
            if ((row && !take_pair(out, "q_row", "s_row", M, K, *x, r)) || (col && !take_pair(out, "q_colT", "s_colT", K, M, *x, c)))
                Py_RETURN_NONE;
        } else {
            if (row) r = {make(M, K, at::kByte, *x), make(M, std::max<int64_t>(K / kGroup, 1), at::kFloat, *x)};
            if (col) c = {make(K, M, at::kByte, *x), make(K, std::max<int64_t>(M / kGroup, 1), at::kFloat, *x)};
        }
        const float* xs = fp8 ? in<float>(*xs_t) : nullptr;
        uint8_t *qr = row ? outp(r.q) : nullptr, *qc = col ? outp(c.q) : nullptr;
        float *sr = row ? outp<float>(r.s) : nullptr, *sc = col ? outp<float>(c.s) : nullptr;
        const void* xp = in(*x);
        void* st = stream();
        jet_status e;
        Py_BEGIN_ALLOW_THREADS
        e = jet_quant_act(xp, xs, fp8 ? JET_SRC_FP8_ROW : JET_SRC_BF16, M, K, qr, sr, qc, sc, st);
        Py_END_ALLOW_THREADS
        return finish(e, "jet_quant_act", e == JET_OK ? same_or(out, row ? &r : nullptr, col ? &c : nullptr) : nullptr);
    });
}

// out: None or a dict that holds the row pair
bool row_pair(PyObject* out, int64_t M, int64_t K, const at::Tensor& like, Pair& r) {
    if (out == Py_None) {
        r = {make(M, K, at::kByte, like), make(M, std::max<int64_t>(K / kGroup, 1), at::kFloat, like)};
        return true;
    }
    return PyDict_CheckExact(out) && take_pair(out, "q_row", "s_row", M, K, like, r);
}

// rmsnorm_quant(x, gamma, eps, out | None)
PyObject* rmsnorm_quant(PyObject*, PyObject* const* a, Py_ssize_t n) {
    if (!args(n, 4)) return nullptr;
    return guarded([&]() -> PyObject* {
        const at::Tensor *x = plain2d(a[0], at::kBFloat16), *g = plain(a[1], at::kBFloat16);
        if (!x || !g || !PyFloat_CheckExact(a[2]) || modes_active()) Py_RETURN_NONE;
        const int64_t M = x->size(0), K = x->size(1);
        if (g->dim() != 1 || g->size(0) != K || !g->is_contiguous() || g->device() != x->device()) Py_RETURN_NONE;
        Pair r;
        if (!row_pair(a[3], M, K, *x, r)) Py_RETURN_NONE;
        const float eps = (float)PyFloat_AS_DOUBLE(a[2]);
        const void *xp = in(*x), *gp = in(*g);
        uint8_t* q = outp(r.q);
        float* s = outp<float>(r.s);
        void* st = stream();
        jet_status e;
        Py_BEGIN_ALLOW_THREADS
        e = jet_rmsnorm_quant(xp, gp, eps, M, K, q, s, st);
        Py_END_ALLOW_THREADS
        return finish(e, "jet_rmsnorm_quant", e == JET_OK ? same_or(a[3], &r, nullptr) : nullptr);
    });
}

// gate and up: bf16 [M, K] on one GPU, of unit column stride and one row stride
bool gate_up(PyObject* const* a, const at::Tensor*& g, const at::Tensor*& u) {
    g = plain(a[0], at::kBFloat16);
    u = plain(a[1], at::kBFloat16);
    return g && u && g->dim() == 2 && u->dim() == 2 && g->stride(1) == 1 && u->stride(1) == 1 &&
           g->sizes() == u->sizes() && g->stride(0) == u->stride(0) && g->device() == u->device();
}

// silu_mul_quant(gate, up, out | None)
PyObject* silu_mul_quant(PyObject*, PyObject* const* a, Py_ssize_t n) {
    if (!args(n, 3)) return nullptr;
    return guarded([&]() -> PyObject* {
        const at::Tensor *g, *u;
        if (!gate_up(a, g, u) || modes_active()) Py_RETURN_NONE;
        const int64_t M = g->size(0), K = g->size(1), ld = g->stride(0);
        Pair r;
        if (!row_pair(a[2], M, K, *g, r)) Py_RETURN_NONE;
        const void *gp = in(*g), *up = in(*u);
        uint8_t* q = outp(r.q);
        float* s = outp<float>(r.s);
        void* st = stream();
        jet_status e;
        Py_BEGIN_ALLOW_THREADS
        e = jet_silu_mul_quant(gp, up, ld, M, K, q, s, st);
        Py_END_ALLOW_THREADS
        return finish(e, "jet_silu_mul_quant", e == JET_OK ? same_or(a[2], &r, nullptr) : nullptr);
    });
}

// silu_mul_bwd(gate, up, dh, out | None)
PyObject* silu_mul_bwd(PyObject*, PyObject* const* a, Py_ssize_t n) {
    if (!args(n, 4)) return nullptr;
    return guarded([&]() -> PyObject* {
        const at::Tensor *g, *u, *dh = plain2d(a[2], at::kBFloat16);
        if (!gate_up(a, g, u) || !dh || dh->sizes() != g->sizes() || dh->device() != g->device() || modes_active()) Py_RETURN_NONE;
        const int64_t M = g->size(0), K = g->size(1), ld = g->stride(0);
        at::Tensor o;
        if (a[3] == Py_None) {
            o = make(M, 2 * K, at::kBFloat16, *g);
        } else {
            const at::Tensor* t = plain2d(a[3], at::kBFloat16);
            if (!t || t->size(0) != M || t->size(1) != 2 * K || t->device() != g->device()) Py_RETURN_NONE;
            o = *t;
        }
        const void *gp = in(*g), *up = in(*u), *dp = in(*dh);
        uint8_t* op = outp(o);
        void* st = stream();
        jet_status e;
        Py_BEGIN_ALLOW_THREADS
        e = jet_silu_mul_bwd(gp, up, ld, dp, M, K, op, op + 2 * K, 2 * K, st);
        Py_END_ALLOW_THREADS
        if (e != JET_OK) return finish(e, "jet_silu_mul_bwd", nullptr);
        if (a[3] == Py_None) return THPVariable_Wrap(o);
        Py_INCREF(a[3]);
        return a[3];
    });
}

// quant_weight(w, transposed, out | None); out: a tuple of 2 or 4 tensors
PyObject* quant_weight(PyObject*, PyObject* const* a, Py_ssize_t n) {
    if (!args(n, 3)) return nullptr;
    return guarded([&]() -> PyObject* {
        const int transposed = PyObject_IsTrue(a[1]);
        if (transposed < 0) return nullptr;
        const at::Tensor* w = plain2d(a[0], at::kBFloat16);
        if (!w || modes_active()) Py_RETURN_NONE;
        const int64_t N = w->size(0), K = w->size(1);
        at::Tensor t[4];
        PyObject* o[4] = {nullptr, nullptr, nullptr, nullptr};
        int have = transposed ? 4 : 2;
        if (a[2] == Py_None) {
            t[0] = make(N, K, at::kByte, *w);
            t[1] = make(std::max<int64_t>(N / kGroup, 1), std::max<int64_t>(K / kGroup, 1), at::kFloat, *w);
            if (transposed) {
                t[2] = make(K, N, at::kByte, *w);
                t[3] = make(std::max<int64_t>(K / kGroup, 1), std::max<int64_t>(N / kGroup, 1), at::kFloat, *w);
            }
        } else {
            // the tuple says what is written, `transposed` what is returned
            if (!PyTuple_CheckExact(a[2])) Py_RETURN_NONE;
            have = (int)PyTuple_GET_SIZE(a[2]);
            if (have != 4 && !(have == 2 && !transposed)) Py_RETURN_NONE;
            for (int i = 0; i < have; ++i) {
                o[i] = PyTuple_GET_ITEM(a[2], i);
                if (!THPVariable_CheckExact(o[i])) Py_RETURN_NONE;
                t[i] = THPVariable_Unpack(o[i]);
            }
            if (!holds(t[0], kCodes, N, K, *w) || !holds(t[1], kScales, N / kGroup, K / kGroup, *w) ||
                (have == 4 && !(holds(t[2], kCodes, K, N, *w) && holds(t[3], kScales, K / kGroup, N / kGroup, *w))))
                Py_RETURN_NONE;
        }
        const void* wp = in(*w);
        uint8_t *q = outp(t[0]), *qT = have == 4 ? outp(t[2]) : nullptr;
        float *s = outp<float>(t[1]), *sT = have == 4 ? outp<float>(t[3]) : nullptr;
        void* st = stream();
        jet_status e;
        Py_BEGIN_ALLOW_THREADS
        e = jet_quant_weight(wp, N, K, q, s, qT, sT, st);
        Py_END_ALLOW_THREADS
        if (e != JET_OK) return finish(e, "jet_quant_weight", nullptr);
        const int ret = transposed ? 4 : 2;
        PyObject* r = PyTuple_New(ret);
        for (int i = 0; r && i < ret; ++i) {
            PyObject* v = o[i];
            if (v) Py_INCREF(v);
            else v = THPVariable_Wrap(t[i]);
            if (!v) {
                Py_DECREF(r);
                return nullptr;
            }
            PyTuple_SET_ITEM(r, i, v);
        }
        return r;
    });
}

// codes [rows, R] with scales [rows / per, R / 128]
bool operand(PyObject* qo, PyObject* so, int64_t per, const at::Tensor*& q, const at::Tensor*& s) {
    q = plain2d(qo, at::kByte);
    s = plain2d(so, at::kFloat);
    if (!q || !s) return false;
    const int64_t rows = q->size(0), R = q->size(1);
    return R % kGroup == 0 && rows % per == 0 && s->size(0) == rows / per && s->size(1) == R / kGroup && s->device() == q->device();
}

// gemm(kind, a, sa, b, sb, out | None): kind 0 FProp, 1 DGrad, 2 WGrad; OUT[i,j] = sum_r A[i,r] B[j,r]
PyObject* gemm(PyObject*, PyObject* const* a, Py_ssize_t n) {
    if (!args(n, 6)) return nullptr;
    return guarded([&]() -> PyObject* {
        const long kind = PyLong_AsLong(a[0]);
        if (kind == -1 && PyErr_Occurred()) return nullptr;
        const at::Tensor *qa, *sa, *qb, *sb;
        if (!operand(a[1], a[2], 1, qa, sa) || !operand(a[3], a[4], kind == 2 ? 1 : kGroup, qb, sb) || modes_active()) Py_RETURN_NONE;
        const int64_t I = qa->size(0), J = qb->size(0), R = qa->size(1);
        if (qb->size(1) != R || qa->device() != qb->device()) Py_RETURN_NONE;
        at::Tensor o;
        if (a[5] == Py_None) {
            o = make(I, J, at::kBFloat16, *qa);
        } else {
            const at::Tensor* t = plain2d(a[5], at::kBFloat16);
            if (!t || t->size(0) != I || t->size(1) != J || t->device() != qa->device()) Py_RETURN_NONE;
            o = *t;
        }
        const uint8_t *pa = in(*qa), *pb = in(*qb);
        const float *psa = in<float>(*sa), *psb = in<float>(*sb);
        void *po = outp(o), *st = stream();
        jet_status e;
        Py_BEGIN_ALLOW_THREADS
        e = kind == 0   ? jet_fp8_linear_fwd(pa, psa, pb, psb, po, I, J, R, st)
            : kind == 1 ? jet_fp8_linear_dgrad(pa, psa, pb, psb, po, I, R, J, st)
                        : jet_fp8_linear_wgrad(pa, psa, pb, psb, po, R, I, J, st);
        Py_END_ALLOW_THREADS
        if (e != JET_OK)
            return finish(e, kind == 0 ? "jet_fp8_linear_fwd" : kind == 1 ? "jet_fp8_linear_dgrad" : "jet_fp8_linear_wgrad", nullptr);
        if (a[5] == Py_None) return THPVariable_Wrap(o);
        Py_INCREF(a[5]);
        return a[5];
    });
}

// ---------------------------------------------------------------- attention

// bf16 [rows, heads, dim] with dense heads, on like's device; a negative size: any.  ld: its row stride
const at::Tensor* heads(PyObject* obj, int64_t rows, int64_t n, int64_t dim, const at::Tensor* like, int64_t& ld) {
    const at::Tensor* t = plain(obj, at::kBFloat16);
    if (!t || t->dim() != 3 || t->stride(2) != 1 || (t->size(1) > 1 && t->stride(1) != t->size(2))) return nullptr;
    if ((rows >= 0 && t->size(0) != rows) || (n >= 0 && t->size(1) != n) || (dim >= 0 && t->size(2) != dim)) return nullptr;
    if (like && t->device() != like->device()) return nullptr;
    const int64_t width = t->size(1) * t->size(2);
    ld = t->size(0) > 1 ? t->stride(0) : width;
    return ld < width ? nullptr : t;
}
const at::Tensor* dense_heads(PyObject* obj, int64_t rows, int64_t n, int64_t dim, const at::Tensor& like) {
    int64_t ld;
    const at::Tensor* t = heads(obj, rows, n, dim, &like, ld);
    return t && ld == n * dim ? t : nullptr;
}
// bf16 [rows, >= cols] of unit column stride
const at::Tensor* wide(PyObject* obj, int64_t cols, int64_t& ld) {
    const at::Tensor* t = plain(obj, at::kBFloat16);
    if (!t || t->dim() != 2 || t->stride(1) != 1 || t->size(1) < cols) return nullptr;
    ld = t->size(0) > 1 ? t->stride(0) : cols;
    return t;
}
// contiguous [n] (negative: any length) on like's device
const at::Tensor* vec(PyObject* obj, at::ScalarType dtype, int64_t n, const at::Tensor& like) {
    const at::Tensor* t = plain(obj, dtype);
    return t && t->dim() == 1 && t->is_contiguous() && (n < 0 || t->size(0) == n) && t->device() == like.device() ? t : nullptr;
}
// New tensors straight from the device's allocator, without the dispatcher in between (0.3 us each)
at::Tensor fresh(at::IntArrayRef sizes, at::ScalarType dtype, const at::Tensor& like) {
    return at::detail::empty_cuda(sizes, dtype, like.device(), std::nullopt);
}
at::Tensor make3(int64_t a, int64_t b, int64_t c, const at::Tensor& like) { return fresh({a, b, c}, at::kBFloat16, like); }
// Scratch memory of one call: back in its stream's pool when the call returns, where only later work of the stream can get it
struct Scratch {
    at::DataPtr p;
    Scratch(int64_t bytes) {
        if (bytes) p = c10::hip::HIPCachingAllocator::get()->allocate((size_t)bytes);
    }
};
// the caching allocator, like the stream, goes by the current device
bool elsewhere(const at::Tensor& t) { return t.device().index() != c10::hip::current_device(); }
bool count(PyObject* obj, int64_t& v) {
    if (!PyLong_CheckExact(obj)) return false;
    v = PyLong_AsLongLong(obj);
    if (v == -1 && PyErr_Occurred()) {
        PyErr_Clear();
        return false;
    }
    return v >= 0 && v < (1 << 30);
}
// whether obj (None where `at` is null) still has its n elements at `at`
bool lies_at(PyObject* obj, const void* at, int64_t n) {
    if (!at || obj == Py_None) return !at && obj == Py_None;
    if (!THPVariable_CheckExact(obj)) return false;
    const at::Tensor& t = THPVariable_Unpack(obj);
    if (!t.is_cuda() || t.numel() != n || !t.is_contiguous()) return false;
    const at::Storage& s = t.storage();
    const size_t first = (size_t)t.storage_offset() * t.itemsize();
    return static_cast<const char*>(s.data()) + first == at && s.nbytes() >= first + (size_t)n * t.itemsize();
}
// the descriptor that a KvCache holds; false: obj is none, lies elsewhere than like, or its tensors were given other memory
bool cache_of(PyObject* obj, const at::Tensor& like, const jet_kv_cache*& desc) {
    if (!PyObject_TypeCheck(obj, reinterpret_cast<PyTypeObject*>(g_cache))) return false;
    PyObject* a = PyObject_GetAttrString(obj, "_where");     // (address of the descriptor, device index, k, v, k_scale, v_scale)
    if (!a) {
        PyErr_Clear();
        return false;
    }
    bool ok = PyTuple_CheckExact(a) && PyTuple_GET_SIZE(a) == 6;
    if (ok) {
        desc = static_cast<const jet_kv_cache*>(PyLong_AsVoidPtr(PyTuple_GET_ITEM(a, 0)));
        const long dev = PyLong_AsLong(PyTuple_GET_ITEM(a, 1));
        if (PyErr_Occurred()) {
            PyErr_Clear();
            ok = false;
        } else {
            ok = desc && dev == like.device().index();
        }
    }
    if (ok) {
        const int64_t rows = desc->n_pages * desc->n_kv * desc->page;
        ok = lies_at(PyTuple_GET_ITEM(a, 2), desc->k, rows * desc->dim) && lies_at(PyTuple_GET_ITEM(a, 3), desc->v, rows * desc->dim) &&
             lies_at(PyTuple_GET_ITEM(a, 4), desc->k_scale, rows) && lies_at(PyTuple_GET_ITEM(a, 5), desc->v_scale, rows);
    }
    Py_DECREF(a);
    return ok;
}
// a new tuple of n tensors; nullptr entries become None
PyObject* tuple_of(const at::Tensor* const* t, int n) {
    PyObject* r = PyTuple_New(n);
    for (int i = 0; r && i < n; ++i) {
        PyObject* v = t[i] ? THPVariable_Wrap(*t[i]) : Py_NewRef(Py_None);
        if (!v) {
            Py_DECREF(r);
            return nullptr;
        }
        PyTuple_SET_ITEM(r, i, v);
    }
    return r;
}

// table, positions, gammas and eps, as both passes of the norm and rotation take them
struct QkShared {
    const at::Tensor *table, *positions, *gq = nullptr, *gk = nullptr;
    int64_t dim;
    float eps;
    bool take(PyObject* const* a, int64_t T, const at::Tensor& like) {   // a: table, positions, gamma_q, gamma_k, eps
        table = plain2d(a[0], at::kFloat);
        if (elsewhere(like) || !table || table->device() != like.device()) return false;
        dim = table->size(1);
        positions = vec(a[1], at::kInt, T, like);
        if (!positions || (a[2] == Py_None) != (a[3] == Py_None) || !PyFloat_CheckExact(a[4])) return false;
        if (a[2] != Py_None) {
            gq = vec(a[2], at::kBFloat16, dim, like);
            gk = vec(a[3], at::kBFloat16, dim, like);
            if (!gq || !gk) return false;
        }
        eps = (float)PyFloat_AS_DOUBLE(a[4]);
        return true;
    }
};
const void* in_or_null(const at::Tensor* t) { return t ? t->const_data_ptr() : nullptr; }

// qk_norm_rope(qkv, n_q, n_kv, table, positions, gamma_q | None, gamma_k | None, eps, cache | None, slots | None)
PyObject* qk_norm_rope(PyObject*, PyObject* const* a, Py_ssize_t n) {
    if (!args(n, 10)) return nullptr;
    return guarded([&]() -> PyObject* {
        int64_t n_q, n_kv, ld;
        const at::Tensor* x = plain(a[0], at::kBFloat16);
        QkShared c;
        if (!x || x->dim() != 2 || !count(a[1], n_q) || !count(a[2], n_kv) || modes_active()) Py_RETURN_NONE;
        const int64_t T = x->size(0);
        if (!c.take(a + 3, T, *x) || !wide(a[0], (n_q + 2 * n_kv) * c.dim, ld) || (a[8] == Py_None) != (a[9] == Py_None)) Py_RETURN_NONE;
        const jet_kv_cache* cache = nullptr;
        const at::Tensor* slots = nullptr;
        if (a[8] != Py_None && (!cache_of(a[8], *x, cache) || !(slots = vec(a[9], at::kLong, T, *x)))) Py_RETURN_NONE;
        const at::Tensor q = make3(T, n_q, c.dim, *x), k = make3(T, n_kv, c.dim, *x);
        const void* xp = in(*x);
        const float* tp = in<float>(*c.table);
        const int64_t rows = c.table->size(0);
        const int32_t* pp = in<int32_t>(*c.positions);
        const int64_t* sp = slots ? in<int64_t>(*slots) : nullptr;
        const void *gq = in_or_null(c.gq), *gk = in_or_null(c.gk);
        void *qp = outp(q), *kp = outp(k), *st = stream();
        jet_status e;
        Py_BEGIN_ALLOW_THREADS
        e = jet_qk_norm_rope(xp, ld, T, n_q, n_kv, c.dim, tp, rows, pp, gq, gk, c.eps, qp, kp, cache, sp, st);
        Py_END_ALLOW_THREADS
        const at::Tensor* r[] = {&q, &k};
        return finish(e, "jet_qk_norm_rope", e == JET_OK ? tuple_of(r, 2) : nullptr);
    });
}

// qk_norm_rope_bwd(dq, dk, qkv | None, table, positions, gamma_q | None, gamma_k | None, eps); a call with `out` is not taken
PyObject* qk_norm_rope_bwd(PyObject*, PyObject* const* a, Py_ssize_t n) {
    if (!args(n, 8)) return nullptr;
    return guarded([&]() -> PyObject* {
        int64_t ld = 0;
        const at::Tensor *dq = plain(a[0], at::kBFloat16), *dk = plain(a[1], at::kBFloat16), *x = nullptr;
        QkShared c;
        if (!dq || !dk || dq->dim() != 3 || dk->dim() != 3 || modes_active()) Py_RETURN_NONE;
        const int64_t T = dq->size(0), n_q = dq->size(1), n_kv = dk->size(1);
        if (!c.take(a + 3, T, *dq) || !dense_heads(a[0], T, n_q, c.dim, *dq) || !dense_heads(a[1], T, n_kv, c.dim, *dq)) Py_RETURN_NONE;
        if (c.gq && (!(x = wide(a[2], (n_q + 2 * n_kv) * c.dim, ld)) || x->size(0) != T || x->device() != dq->device())) Py_RETURN_NONE;
        const at::Tensor dx = fresh({T, (n_q + n_kv) * c.dim}, at::kBFloat16, *dq);
        at::Tensor gq, gk;
        if (c.gq) {
            gq = fresh({c.dim}, at::kFloat, *dq);
            gk = fresh({c.dim}, at::kFloat, *dq);
        }
        const Scratch ws(c.gq ? jet_qk_norm_rope_bwd_workspace(T, n_q, n_kv, c.dim) : 0);
        const void *dqp = in(*dq), *dkp = in(*dk), *xp = in_or_null(x), *gqp = in_or_null(c.gq), *gkp = in_or_null(c.gk);
        const float* tp = in<float>(*c.table);
        const int64_t rows = c.table->size(0);
        const int32_t* pp = in<int32_t>(*c.positions);
        float *ogq = c.gq ? outp<float>(gq) : nullptr, *ogk = c.gq ? outp<float>(gk) : nullptr;
        void *dxp = outp(dx), *wsp = ws.p.get(), *st = stream();
        jet_status e;
        Py_BEGIN_ALLOW_THREADS
        e = jet_qk_norm_rope_bwd(dqp, dkp, xp, ld, T, n_q, n_kv, c.dim, tp, rows, pp, gqp, gkp, c.eps, dxp, (n_q + n_kv) * c.dim, ogq, ogk, wsp, st);
        Py_END_ALLOW_THREADS
        const at::Tensor* r[] = {&dx, c.gq ? &gq : nullptr, c.gq ? &gk : nullptr};
        return finish(e, "jet_qk_norm_rope_bwd", e == JET_OK ? tuple_of(r, 3) : nullptr);
    });
}

// q, k, v, cu_q, cu_k | None, causal, scale | None, as both passes over packed sequences take them
struct Packed {
    const at::Tensor *q, *k, *v, *cq, *ck;
    int64_t ldq, ldk, ldv, Tq, Tk, n_q, n_kv, dim, n_seqs;
    int causal;
    float scale;
    bool take(PyObject* const* qkv, PyObject* const* rest) {
        q = heads(qkv[0], -1, -1, -1, nullptr, ldq);
        if (!q || elsewhere(*q)) return false;
        Tq = q->size(0), n_q = q->size(1), dim = q->size(2);
        k = heads(qkv[1], -1, -1, dim, q, ldk);
        if (!k) return false;
        Tk = k->size(0), n_kv = k->size(1);
        v = heads(qkv[2], Tk, n_kv, dim, q, ldv);
        cq = vec(rest[0], at::kInt, -1, *q);
        if (!v || !cq) return false;
        ck = rest[1] == Py_None ? cq : vec(rest[1], at::kInt, cq->size(0), *q);
        n_seqs = cq->size(0) - 1;
        causal = rest[2] == Py_True;
        if (!ck || !PyBool_Check(rest[2])) return false;
        return softmax_scale(rest[3], dim, scale);
    }
    static bool softmax_scale(PyObject* o, int64_t dim, float& scale) {
        if (o != Py_None && !PyFloat_CheckExact(o)) return false;
        scale = o == Py_None ? (float)(1.0 / std::sqrt((double)dim)) : (float)PyFloat_AS_DOUBLE(o);
        return true;
    }
};

// attention_fwd(q, k, v, cu_q, cu_k | None, causal, scale | None)
PyObject* attention_fwd(PyObject*, PyObject* const* a, Py_ssize_t n) {
    if (!args(n, 7)) return nullptr;
    return guarded([&]() -> PyObject* {
        Packed c;
        if (modes_active() || !c.take(a, a + 3)) Py_RETURN_NONE;
        const at::Tensor o = make3(c.Tq, c.n_q, c.dim, *c.q), lse = fresh({c.n_q, c.Tq}, at::kFloat, *c.q);
        const void *qp = in(*c.q), *kp = in(*c.k), *vp = in(*c.v);
        const int32_t *cq = in<int32_t>(*c.cq), *ck = in<int32_t>(*c.ck);
        float* lp = outp<float>(lse);
        void *op = outp(o), *st = stream();
        jet_status e;
        Py_BEGIN_ALLOW_THREADS
        e = jet_attention_fwd(qp, c.ldq, kp, c.ldk, vp, c.ldv, cq, ck, c.n_seqs, c.Tq, c.Tk, c.n_q, c.n_kv, c.dim, c.scale, c.causal, op, lp, st);
        Py_END_ALLOW_THREADS
        const at::Tensor* r[] = {&o, &lse};
        return finish(e, "jet_attention_fwd", e == JET_OK ? tuple_of(r, 2) : nullptr);
    });
}

// attention_bwd(q, k, v, o, lse, do, cu_q, cu_k | None, causal, scale | None); a call with `out` is not taken
PyObject* attention_bwd(PyObject*, PyObject* const* a, Py_ssize_t n) {
    if (!args(n, 10)) return nullptr;
    return guarded([&]() -> PyObject* {
        Packed c;
        if (modes_active() || !c.take(a, a + 6)) Py_RETURN_NONE;
        const at::Tensor *o = dense_heads(a[3], c.Tq, c.n_q, c.dim, *c.q), *lse = plain2d(a[4], at::kFloat),
                         *dout = dense_heads(a[5], c.Tq, c.n_q, c.dim, *c.q);
        if (!o || !lse || !dout || lse->size(0) != c.n_q || lse->size(1) != c.Tq || lse->device() != c.q->device()) Py_RETURN_NONE;
        const at::Tensor dq = make3(c.Tq, c.n_q, c.dim, *c.q), dk = make3(c.Tk, c.n_kv, c.dim, *c.q), dv = make3(c.Tk, c.n_kv, c.dim, *c.q);
        const Scratch ws(jet_attention_bwd_workspace(c.n_seqs, c.Tq, c.Tk, c.n_q, c.n_kv, c.dim));
        const void *qp = in(*c.q), *kp = in(*c.k), *vp = in(*c.v), *op = in(*o), *dp = in(*dout);
        const float* lp = in<float>(*lse);
        const int32_t *cq = in<int32_t>(*c.cq), *ck = in<int32_t>(*c.ck);
        void *dqp = outp(dq), *dkp = outp(dk), *dvp = outp(dv), *wp = ws.p.get(), *st = stream();
        jet_status e;
        Py_BEGIN_ALLOW_THREADS
        e = jet_attention_bwd(qp, c.ldq, kp, c.ldk, vp, c.ldv, op, lp, dp, cq, ck, c.n_seqs, c.Tq, c.Tk, c.n_q, c.n_kv, c.dim, c.scale, c.causal,
                              dqp, c.n_q * c.dim, dkp, c.n_kv * c.dim, dvp, c.n_kv * c.dim, wp, st);
        Py_END_ALLOW_THREADS
        const at::Tensor* r[] = {&dq, &dk, &dv};
        return finish(e, "jet_attention_bwd", e == JET_OK ? tuple_of(r, 3) : nullptr);
    });
}

// attention_decode(q, cache, pages, lengths, scale | None)
PyObject* attention_decode(PyObject*, PyObject* const* a, Py_ssize_t n) {
    if (!args(n, 5)) return nullptr;
    return guarded([&]() -> PyObject* {
        int64_t ld;
        const at::Tensor* q = heads(a[0], -1, -1, -1, nullptr, ld);
        const at::Tensor* pages = plain2d(a[2], at::kInt);
        const jet_kv_cache* cache = nullptr;
        if (!q || elsewhere(*q) || !pages || modes_active() || !cache_of(a[1], *q, cache)) Py_RETURN_NONE;
        const int64_t B = q->size(0), n_q = q->size(1), dim = q->size(2), max_pages = pages->size(1);
        const at::Tensor* lengths = vec(a[3], at::kInt, B, *q);
        float scale;
        if (!lengths || pages->size(0) != B || pages->device() != q->device() || cache->dim != dim || !Packed::softmax_scale(a[4], dim, scale))
            Py_RETURN_NONE;
        const at::Tensor o = make3(B, n_q, dim, *q);
        const Scratch ws(jet_attention_decode_workspace(cache, B, n_q, max_pages));
        const void* qp = in(*q);
        const int32_t *pp = in<int32_t>(*pages), *lp = in<int32_t>(*lengths);
        void *op = outp(o), *wp = ws.p.get(), *st = stream();
        jet_status e;
        Py_BEGIN_ALLOW_THREADS
        e = jet_attention_decode(qp, ld, n_q, cache, pp, max_pages, lp, B, scale, op, wp, st);
        Py_END_ALLOW_THREADS
        return finish(e, "jet_attention_decode", e == JET_OK ? THPVariable_Wrap(o) : nullptr);
    });
}

// init(JetError, torch.OutOfMemoryError, KvCache)
PyObject* init(PyObject*, PyObject* const* a, Py_ssize_t n) {
    if (!args(n, 3)) return nullptr;
    if (!PyType_Check(a[2])) {
        PyErr_SetString(PyExc_TypeError, "KvCache: need a class");
        return nullptr;
    }
    PyObject** const to[] = {&g_error, &g_oom, &g_cache};
    for (int i = 0; i < 3; ++i) {
        Py_INCREF(a[i]);
        Py_XDECREF(*to[i]);
        *to[i] = a[i];
    }
    Py_RETURN_NONE;
}

#define JET_FAST(f) reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(f)), METH_FASTCALL, nullptr
PyMethodDef kMethods[] = {{"init", JET_FAST(init)},
                          {"quant_act", JET_FAST(quant_act)},
                          {"rmsnorm_quant", JET_FAST(rmsnorm_quant)},
                          {"silu_mul_quant", JET_FAST(silu_mul_quant)},
                          {"silu_mul_bwd", JET_FAST(silu_mul_bwd)},
                          {"quant_weight", JET_FAST(quant_weight)},
                          {"gemm", JET_FAST(gemm)},
                          {"qk_norm_rope", JET_FAST(qk_norm_rope)},
                          {"qk_norm_rope_bwd", JET_FAST(qk_norm_rope_bwd)},
                          {"attention_fwd", JET_FAST(attention_fwd)},
                          {"attention_bwd", JET_FAST(attention_bwd)},
                          {"attention_decode", JET_FAST(attention_decode)},
                          {nullptr, nullptr, 0, nullptr}};
PyModuleDef kModule = {PyModuleDef_HEAD_INIT, "_jet_host", nullptr, -1, kMethods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__jet_host() { return PyModule_Create(&kModule); }
