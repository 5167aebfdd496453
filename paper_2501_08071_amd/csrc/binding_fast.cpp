// The Python entry points' way to the C ABI for the usual call: torch tensors on the GPU, right shapes, right types.
//
// A small launch takes the GPU 3 to 6 us.  Looking at each tensor from Python (dtype, shape, contiguity, address), asking torch
// for the current stream and the ctypes call took 7.2 to 9.8 us (row softmax to product), so the host was what such a call waited
// for; from here it is 3.2 to 3.4, the launch itself most of it.  Every function takes the arguments of its namesake in binding.py and returns its result,
// or None for anything out of the ordinary -- whatever is not exactly a tensor with memory of its own on the GPU, a wrong shape
// or type, a status other than 0 (nothing has been launched then) -- and binding.py goes through its own checks, which say what
// is wrong.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <ATen/core/Tensor.h>
#include <ATen/ops/empty.h>
#include <ATen/PythonTorchFunctionTLS.h>
#include <c10/hip/HIPCachingAllocator.h>
#include <c10/hip/HIPGuard.h>
#include <c10/hip/HIPStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include <climits>
#include <initializer_list>

#include "../../include/attn.h"
#include "../../include/gemm.h"
#include "../../include/rowops.h"

namespace {

// the entry points of the library that binding.py has loaded
struct {
    decltype(&attn_fwd) attn;
    decltype(&attn_fwd_o16) attn_o16;
    decltype(&softmax_rows_fwd) softmax;
    decltype(&rmsnorm_fwd) rmsnorm;
    decltype(&gemm_leakyrelu_fwd) gemm;
    decltype(&residual_rmsnorm_fwd) residual_norm;
    decltype(&attn_kv_append) append;
    decltype(&attn_paged_fwd) paged;
    decltype(&attn_paged_workspace) paged_workspace;
} abi;

// A contiguous GPU tensor with memory of its own, or null.
const at::Tensor* gpu_tensor(PyObject* o) {
    if (!THPVariable_CheckExact(o)) return nullptr;
    const at::Tensor& t = THPVariable_Unpack(o);
    return t.defined() && t.has_storage() && t.is_cuda() && t.layout() == at::kStrided && t.is_contiguous() ? &t : nullptr;
}
int type_of(const at::Tensor& t) {
    const auto s = t.scalar_type();
    return s == at::kHalf ? 0 : s == at::kBFloat16 ? 1 : -1;
}
bool fits_int(int64_t n) { return n <= INT_MAX; }
// a plain number as Python's float() and int() would take it
bool real(PyObject* o, double& x) {
    if (!PyFloat_CheckExact(o) && !PyLong_CheckExact(o)) return false;
    x = PyFloat_AsDouble(o);
    return !(x == -1.0 && PyErr_Occurred());
}
bool flag(PyObject* o, int& x) {
    if (!PyBool_Check(o) && !PyLong_CheckExact(o)) return false;
    x = PyObject_IsTrue(o);
    return true;
}
// Where a call goes: the torch stream given, or the current one on t's device.
struct Where {
    void* handle;
    bool elsewhere;             // not the current stream
    c10::DeviceIndex device;
};
bool stream_of(PyObject* o, const at::Tensor& t, Where& w) {
    w.device = t.device().index();
    w.handle = c10::hip::getCurrentHIPStream(w.device).stream();
    w.elsewhere = false;
    if (o == Py_None) return true;
    PyObject* h = PyObject_GetAttrString(o, "cuda_stream");
    if (h == nullptr) return false;
    void* given = PyLong_AsVoidPtr(h);
    Py_DECREF(h);
    if (PyErr_Occurred()) return false;
    w.elsewhere = given != w.handle;
    w.handle = given;
    return true;
}

// Launching and allocating may wait for the GPU, and what the GPU waits for may be Python's (a host function in a stream):
// both run without the interpreter's lock, as a call by way of ctypes does.
struct NoLock {
    PyThreadState* s = PyEval_SaveThread();
    ~NoLock() { PyEval_RestoreThread(s); }
};
// Memory that a call on w writes, for another stream than the current one from that stream's own pool: what is free in the current one's may
// still be written by work under way there, for which the other does not wait.  A result (`returned`) is then told of the current stream, where it
// is likely to be read: it is not handed out again before that is done.
at::Tensor new_tensor(at::IntArrayRef sizes, const at::TensorOptions& opt, const Where& w, bool returned = true) {
    NoLock _;
    if (!w.elsewhere) return at::empty(sizes, opt.requires_grad(false));
    const auto current = c10::hip::getCurrentHIPStream(w.device);
    at::Tensor t;
    {
        c10::hip::HIPStreamGuard there(c10::hip::getStreamFromExternal((hipStream_t)w.handle, w.device));
        t = at::empty(sizes, opt.requires_grad(false));
    }
    if (returned) c10::hip::HIPCachingAllocator::recordStream(t.storage().data_ptr(), current);
    return t;
}

// What any of the functions below may throw (memory for an output, a device that is gone) is left to binding.py's own way.
template <class F>
PyObject* guarded(Py_ssize_t given, Py_ssize_t wanted, F f) {
    if (given != wanted) {
        PyErr_SetString(PyExc_TypeError, "wrong number of arguments");
        return nullptr;
    }
    PyObject* r = nullptr;
    try {
        if (!at::impl::torch_function_mode_enabled()) r = f();
    } catch (...) {
        r = nullptr;
    }
    if (r != nullptr) return r;
    PyErr_Clear();
    Py_RETURN_NONE;
}

template <class F, class... T>
bool launched(F call, const T&... t) {
    return [&](auto... p) {
        NoLock _;
        return call(p...) == 0;
    }(t.mutable_data_ptr()...);
}

// (q, k, v, causal, scale, o, lse, stream, want_lse, o16) -> (o, lse)
PyObject* fast_attn(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded(n, 10, [&]() -> PyObject* {
        const at::Tensor *q = gpu_tensor(a[0]), *k = gpu_tensor(a[1]), *v = gpu_tensor(a[2]);
        if (!q || !k || !v) return nullptr;
        const int dt = type_of(*q);
        if (dt < 0 || type_of(*k) != dt || type_of(*v) != dt || q->dim() != 4 || k->sizes() != q->sizes() || v->sizes() != q->sizes()) return nullptr;
        const auto z = q->sizes();
        if (!fits_int(z[0]) || !fits_int(z[1]) || !fits_int(z[2]) || !fits_int(z[3])) return nullptr;
        int causal, want_lse, o16, rc;
        double scale;
        Where w;
        if (!flag(a[3], causal) || !real(a[4], scale) || !flag(a[8], want_lse) || !flag(a[9], o16) || !stream_of(a[7], *q, w)) return nullptr;
        const auto odt = o16 ? q->scalar_type() : at::kFloat;
        at::Tensor o_new, lse_new;
        const at::Tensor *o, *lse = nullptr;
        if (a[5] == Py_None) o = &(o_new = new_tensor(z, q->options().dtype(odt), w));
        else if (!(o = gpu_tensor(a[5])) || o->scalar_type() != odt || o->sizes() != z) return nullptr;
        if (a[6] != Py_None) {
            if (!(lse = gpu_tensor(a[6])) || lse->scalar_type() != at::kFloat || lse->sizes() != z.slice(0, 3)) return nullptr;
        } else if (want_lse) {
            lse = &(lse_new = new_tensor(z.slice(0, 3), q->options().dtype(at::kFloat), w));
        }
        float* l = lse ? (float*)lse->mutable_data_ptr() : nullptr;
        const int B = (int)z[0], H = (int)z[1], S = (int)z[2], D = (int)z[3];
        const void *qp = q->mutable_data_ptr(), *kp = k->mutable_data_ptr(), *vp = v->mutable_data_ptr();
        void* op = o->mutable_data_ptr();
        {
            NoLock _;
            rc = o16 ? abi.attn_o16(qp, kp, vp, op, l, B, H, S, D, causal, (float)scale, dt, w.handle)
                     : abi.attn(qp, kp, vp, (float*)op, l, B, H, S, D, causal, (float)scale, dt, w.handle);
        }
        if (rc != 0) return nullptr;
        PyObject* po = a[5] != Py_None ? Py_NewRef(a[5]) : THPVariable_Wrap(o_new);
        PyObject* pl = lse_new.defined() ? THPVariable_Wrap(lse_new) : Py_NewRef(a[6]);
        PyObject* r = po && pl ? PyTuple_Pack(2, po, pl) : nullptr;
        Py_XDECREF(po);
        Py_XDECREF(pl);
        return r;
    });
}

// x [..., d] and y of its shape and type (allocated if None); the rows, and where to
const at::Tensor* row_operands(PyObject* px, PyObject* py, PyObject* ps, at::Tensor& y_new, const at::Tensor*& y, long long& rows, int& d, int& dt, Where& w) {
    const at::Tensor* x = gpu_tensor(px);
    if (!x || (dt = type_of(*x)) < 0 || x->dim() < 1 || !stream_of(ps, *x, w)) return nullptr;
    const int64_t n = x->sizes().back();
    if (!fits_int(n)) return nullptr;
    if (py == Py_None) y = &(y_new = new_tensor(x->sizes(), x->options(), w));
    else if (!(y = gpu_tensor(py)) || y->scalar_type() != x->scalar_type() || y->sizes() != x->sizes()) return nullptr;
    d = (int)n;
    rows = n ? x->numel() / n : 0;
    return x;
}
PyObject* given_or_new(PyObject* given, const at::Tensor& fresh) { return given != Py_None ? Py_NewRef(given) : THPVariable_Wrap(fresh); }

// (x, y, stream) -> y
PyObject* fast_softmax(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded(n, 3, [&]() -> PyObject* {
        at::Tensor y_new;
        const at::Tensor* y;
        long long rows;
        int d, dt;
        Where s;
        const at::Tensor* x = row_operands(a[0], a[1], a[2], y_new, y, rows, d, dt, s);
        if (!x) return nullptr;
        if (launched([&](void* xp, void* yp) { return abi.softmax(xp, yp, rows, d, dt, s.handle); }, *x, *y)) return given_or_new(a[1], y_new);
        return nullptr;
    });
}

// (x, w, eps, y, stream) -> y
PyObject* fast_rmsnorm(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded(n, 5, [&]() -> PyObject* {
        at::Tensor y_new;
        const at::Tensor* y;
        long long rows;
        int d, dt;
        Where s;
        double eps;
        const at::Tensor *x = row_operands(a[0], a[3], a[4], y_new, y, rows, d, dt, s), *w = gpu_tensor(a[1]);
        if (!x || !w || w->scalar_type() != x->scalar_type() || w->dim() != 1 || w->sizes()[0] != d) return nullptr;
        if (!real(a[2], eps)) return nullptr;
        if (launched([&](void* xp, void* wp, void* yp) { return abi.rmsnorm(xp, wp, yp, rows, d, (float)eps, dt, s.handle); }, *x, *w, *y))
            return given_or_new(a[3], y_new);
        return nullptr;
    });
}

// (a, b, slope, c, stream) -> c
PyObject* fast_gemm(PyObject*, PyObject* const* g, Py_ssize_t n) {
    return guarded(n, 5, [&]() -> PyObject* {
        const at::Tensor *a = gpu_tensor(g[0]), *b = gpu_tensor(g[1]), *c;
        if (!a || !b) return nullptr;
        const int dt = type_of(*a);
        const int64_t dim = a->dim();
        if (dt < 0 || type_of(*b) != dt || b->dim() != dim || (dim != 2 && dim != 3)) return nullptr;
        const int64_t batch = dim == 3 ? a->size(0) : 1, M = a->size(dim - 2), K = a->size(dim - 1), N = b->size(dim - 1);
        if ((dim == 3 && b->size(0) != batch) || b->size(dim - 2) != K) return nullptr;
        if (!fits_int(batch) || !fits_int(M) || !fits_int(K) || !fits_int(N)) return nullptr;
        double slope;
        Where w;
        if (!real(g[2], slope) || !stream_of(g[4], *a, w)) return nullptr;
        const int64_t shape3[3] = {batch, M, N};
        const at::IntArrayRef shape(shape3 + (3 - dim), dim);
        at::Tensor c_new;
        if (g[3] == Py_None) c = &(c_new = new_tensor(shape, a->options(), w));
        else if (!(c = gpu_tensor(g[3])) || c->scalar_type() != a->scalar_type() || c->sizes() != shape) return nullptr;
        if (launched([&](void* ap, void* bp, void* cp) { return abi.gemm(ap, bp, cp, (int)batch, (int)M, (int)N, (int)K, (float)slope, dt, w.handle); }, *a, *b, *c))
            return given_or_new(g[3], c_new);
        return nullptr;
    });
}

// x, r (or None), w, r_out (allocated if None, and only with r); y is the caller's
struct NormOperands {
    const at::Tensor *x, *r = nullptr, *w, *r_out = nullptr;
    at::Tensor r_new;
    long long rows;
    int d, dt;
    double eps;
    Where st;
    bool take(PyObject* px, PyObject* pr, PyObject* pw, PyObject* pe, PyObject* po, PyObject* ps) {
        x = gpu_tensor(px), w = gpu_tensor(pw);
        if (!x || !w || (dt = type_of(*x)) < 0 || x->dim() < 1 || !real(pe, eps) || !stream_of(ps, *x, st)) return false;
        const int64_t n = x->sizes().back();
        if (!fits_int(n) || w->scalar_type() != x->scalar_type() || w->dim() != 1 || w->sizes()[0] != n) return false;
        d = (int)n;
        rows = n ? x->numel() / n : 0;
        if (pr == Py_None) return true;
        auto like_x = [&](const at::Tensor* t) { return t && t->scalar_type() == x->scalar_type() && t->sizes() == x->sizes(); };
        if (!like_x(r = gpu_tensor(pr))) return false;
        if (po == Py_None) r_out = &(r_new = new_tensor(x->sizes(), x->options(), st));
        else if (!like_x(r_out = gpu_tensor(po))) return false;
        return true;
    }
    bool launch(const at::Tensor& y, const at::Tensor* scale, int group) const {
        void *xp = x->mutable_data_ptr(), *rp = r ? r->mutable_data_ptr() : nullptr, *wp = w->mutable_data_ptr(), *yp = y.mutable_data_ptr(),
             *sp = scale ? scale->mutable_data_ptr() : nullptr, *op = r ? r_out->mutable_data_ptr() : nullptr;
        NoLock _;
        return abi.residual_norm(xp, rp, wp, yp, (float*)sp, op, rows, d, (float)eps, dt, scale != nullptr, group, st.handle) == 0;
    }
    PyObject* r_result(PyObject* given) const { return r ? given_or_new(given, r_new) : Py_NewRef(Py_None); }
};
PyObject* tuple_of(std::initializer_list<PyObject*> items) {
    PyObject* t = PyTuple_New((Py_ssize_t)items.size());
    Py_ssize_t i = 0;
    bool ok = t != nullptr;
    for (PyObject* o : items) {
        ok = ok && o;
        if (t) PyTuple_SET_ITEM(t, i++, o);
        else Py_XDECREF(o);
    }
    if (!ok) Py_CLEAR(t);
    return t;
}

// (x, r, w, eps, y, r_out, stream) -> (y, r_out)
PyObject* fast_residual_norm(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded(n, 7, [&]() -> PyObject* {
        NormOperands o;
        at::Tensor y_new;
        const at::Tensor* y;
        if (!o.take(a[0], a[1], a[2], a[3], a[5], a[6])) return nullptr;
        if (a[4] == Py_None) y = &(y_new = new_tensor(o.x->sizes(), o.x->options(), o.st));
        else if (!(y = gpu_tensor(a[4])) || y->scalar_type() != o.x->scalar_type() || y->sizes() != o.x->sizes()) return nullptr;
        if (!o.launch(*y, nullptr, 0)) return nullptr;
        return tuple_of({given_or_new(a[4], y_new), o.r_result(a[5])});
    });
}

// (x, r, w, eps, group, y, scale, r_out, stream) -> (y, scale, r_out)
PyObject* fast_residual_norm_fp8(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded(n, 9, [&]() -> PyObject* {
        NormOperands o;
        at::Tensor y_new, s_new;
        const at::Tensor *y, *s;
        if (!PyLong_CheckExact(a[4]) || !o.take(a[0], a[1], a[2], a[3], a[7], a[8])) return nullptr;
        const long group = PyLong_AsLong(a[4]);
        if (group != 0 && group != 128) return nullptr;
        if (a[5] == Py_None) y = &(y_new = new_tensor(o.x->sizes(), o.x->options().dtype(at::kFloat8_e4m3fn), o.st));
        else if (!(y = gpu_tensor(a[5])) || y->scalar_type() != at::kFloat8_e4m3fn || y->sizes() != o.x->sizes()) return nullptr;
        c10::SmallVector<int64_t, 6> shape(o.x->sizes().begin(), o.x->sizes().end());
        shape.back() = group ? (o.d + group - 1) / group : 1;
        if (a[6] == Py_None) s = &(s_new = new_tensor(shape, o.x->options().dtype(at::kFloat), o.st));
        else if (!(s = gpu_tensor(a[6])) || s->scalar_type() != at::kFloat || s->sizes() != at::IntArrayRef(shape)) return nullptr;
        if (!o.launch(*y, s, (int)group)) return nullptr;
        return tuple_of({given_or_new(a[5], y_new), given_or_new(a[6], s_new), o.r_result(a[7])});
    });
}

// A GPU tensor with memory of its own, contiguous or not, or null.
const at::Tensor* any_gpu_tensor(PyObject* o) {
    if (!THPVariable_CheckExact(o)) return nullptr;
    const at::Tensor& t = THPVariable_Unpack(o);
    return t.defined() && t.has_storage() && t.is_cuda() && t.layout() == at::kStrided ? &t : nullptr;
}
// [T, heads, D], a token's heads contiguous, all sizes at least 1
const at::Tensor* heads_of(PyObject* o) {
    const at::Tensor* t = any_gpu_tensor(o);
    if (!t || t->dim() != 3 || t->numel() == 0) return nullptr;
    return t->stride(2) == 1 && (t->stride(1) == t->size(2) || t->size(1) == 1) ? t : nullptr;
}
const at::Tensor* ints(PyObject* o, int dim) {
    const at::Tensor* t = any_gpu_tensor(o);
    return t && t->scalar_type() == at::kInt && t->dim() == dim && t->numel() > 0 && t->stride(dim - 1) == 1 ? t : nullptr;
}
bool whole(PyObject* o, int& x) {
    if (!PyLong_CheckExact(o)) return false;
    const long v = PyLong_AsLong(o);
    if ((v == -1 && PyErr_Occurred()) || v < INT_MIN || v > INT_MAX) return false;
    x = (int)v;
    return true;
}
// k_cache, v_cache, page_table, cu_q, kv_len in a row at `a`, for T tokens
bool cache_of(PyObject* const* a, int64_t T, attn_paged_t& c, at::ScalarType& type) {
    const at::Tensor *k = any_gpu_tensor(a[0]), *v = any_gpu_tensor(a[1]), *table = ints(a[2], 2), *cu = ints(a[3], 1), *len = ints(a[4], 1);
    if (!k || !v || !table || !cu || !len) return false;
    type = k->scalar_type();
    c.dtype = type_of(*k);
    if (c.dtype < 0 || v->scalar_type() != type || k->dim() != 4 || v->sizes() != k->sizes() || v->strides() != k->strides() || k->numel() == 0) return false;
    const auto z = k->sizes(), s = k->strides();
    if (s[3] != 1 || s[2] != z[3] || s[1] != z[2] * z[3] || s[0] < z[1] * z[2] * z[3]) return false;
    const int64_t B = len->size(0);
    if (cu->size(0) != B + 1 || table->size(0) != B || !fits_int(z[0]) || !fits_int(z[1]) || !fits_int(z[2]) || !fits_int(z[3]) || !fits_int(B) ||
        !fits_int(T) || !fits_int(table->size(1)) || !fits_int(table->stride(0)))
        return false;
    c.k = k->mutable_data_ptr(), c.v = v->mutable_data_ptr();
    c.page_stride = s[0];
    c.n_pages = (int)z[0], c.Hk = (int)z[1], c.page_size = (int)z[2], c.D = (int)z[3];
    c.page_table = (const int*)table->mutable_data_ptr();
    c.table_stride = B > 1 ? (int)table->stride(0) : (int)table->size(1), c.width = (int)table->size(1);
    c.cu_q = (const int*)cu->mutable_data_ptr(), c.kv_len = (const int*)len->mutable_data_ptr();
    c.B = (int)B, c.T = (int)T;
    return true;
}
int64_t token_stride(const at::Tensor& t) { return t.size(0) > 1 ? t.stride(0) : t.size(1) * t.size(2); }

// (q, k, v, k_cache, v_cache, page_table, cu_q, kv_len, cos, sin, interleaved, pos_offset, q_out, stream) -> q_out
PyObject* fast_append(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded(n, 14, [&]() -> PyObject* {
        const at::Tensor *q = heads_of(a[0]), *k = heads_of(a[1]), *v = heads_of(a[2]), *cos = nullptr, *sin = nullptr, *out;
        attn_paged_t c;
        at::ScalarType type;
        if (!q || !k || !v || !cache_of(a + 3, k->size(0), c, type)) return nullptr;
        for (const at::Tensor* t : {q, k, v})
            if (t->scalar_type() != type || t->size(0) != c.T || t->size(2) != c.D) return nullptr;
        if (k->size(1) != c.Hk || v->size(1) != c.Hk || !fits_int(q->size(1))) return nullptr;
        int interleaved, offset, rot = 0, angles = 0;
        Where w;
        if (!flag(a[10], interleaved) || !whole(a[11], offset) || !stream_of(a[13], *k, w)) return nullptr;
        if (a[8] != Py_None || a[9] != Py_None) {
            cos = gpu_tensor(a[8]), sin = gpu_tensor(a[9]);
            if (!cos || !sin || cos->scalar_type() != at::kFloat || sin->scalar_type() != at::kFloat || cos->dim() != 2 || sin->sizes() != cos->sizes()) return nullptr;
            if (!fits_int(cos->size(0)) || cos->size(1) > c.D) return nullptr;
            angles = (int)cos->size(0), rot = 2 * (int)cos->size(1);
        }
        at::Tensor fresh;
        if (a[12] == Py_None) out = &(fresh = new_tensor(q->sizes(), q->options(), w));
        else if (!(out = gpu_tensor(a[12])) || out->scalar_type() != type || out->sizes() != q->sizes()) return nullptr;
        const int64_t qs = token_stride(*q), ks = token_stride(*k), vs = token_stride(*v);
        const int Hq = (int)q->size(1);
        const void *qp = q->mutable_data_ptr(), *kp = k->mutable_data_ptr(), *vp = v->mutable_data_ptr();
        const float *cp = cos ? (const float*)cos->mutable_data_ptr() : nullptr, *sp = sin ? (const float*)sin->mutable_data_ptr() : nullptr;
        void* op = out->mutable_data_ptr();
        int rc;
        {
            NoLock _;
            rc = abi.append(&c, qp, kp, vp, qs, ks, vs, op, cp, sp, rot, interleaved, angles, offset, Hq, w.handle);
        }
        return rc == 0 ? given_or_new(a[12], fresh) : nullptr;
    });
}

// (q, k_cache, v_cache, page_table, cu_q, kv_len, scale, max_q, max_kv, prefix_table, prefix_len, o, lse, stream, want_lse, workspace) -> (o, lse)
PyObject* fast_paged(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded(n, 16, [&]() -> PyObject* {
        const at::Tensor *q = heads_of(a[0]), *o, *lse = nullptr, *ws, *prefix = nullptr;
        attn_paged_t c;
        at::ScalarType type;
        double scale;
        int max_q, max_kv, prefix_len, want_lse;
        Where w;
        if (!q || !cache_of(a + 1, q->size(0), c, type) || q->scalar_type() != type || q->size(2) != c.D || !fits_int(q->size(1))) return nullptr;
        if (!real(a[6], scale) || !whole(a[10], prefix_len) || !flag(a[14], want_lse) || !stream_of(a[13], *q, w)) return nullptr;
        if (a[7] == Py_None) max_q = c.T;
        else if (!whole(a[7], max_q)) return nullptr;
        if (a[8] == Py_None) {
            const int64_t all = (int64_t)c.width * c.page_size;
            if (!fits_int(all)) return nullptr;
            max_kv = (int)all;
        } else if (!whole(a[8], max_kv)) return nullptr;
        if (prefix_len != 0 && (prefix_len < 0 || !(prefix = ints(a[9], 1)) || prefix->size(0) * c.page_size < prefix_len)) return nullptr;
        const int Hq = (int)q->size(1);
        const int64_t sizes[3] = {c.T, Hq, c.D};
        at::Tensor o_new, lse_new, ws_new;
        if (a[11] == Py_None) o = &(o_new = new_tensor(sizes, q->options(), w));
        else if (!(o = gpu_tensor(a[11])) || o->scalar_type() != type || o->sizes() != q->sizes()) return nullptr;
        if (a[12] != Py_None) {
            if (!(lse = gpu_tensor(a[12])) || lse->scalar_type() != at::kFloat || lse->sizes() != q->sizes().slice(0, 2)) return nullptr;
        } else if (want_lse) {
            lse = &(lse_new = new_tensor(q->sizes().slice(0, 2), q->options().dtype(at::kFloat), w));
        }
        int64_t bytes = abi.paged_workspace(c.B, c.T, Hq, c.Hk, c.D, max_q, max_kv, prefix_len);
        if (bytes < 0) return nullptr;
        if (a[15] == Py_None) ws = &(ws_new = new_tensor(bytes, q->options().dtype(at::kByte), w, false));
        else if (!(ws = gpu_tensor(a[15])) || ws->scalar_type() != at::kByte) return nullptr;
        bytes = ws->numel();
        const void *qp = q->mutable_data_ptr(), *pp = prefix ? prefix->mutable_data_ptr() : nullptr;
        void *op = o->mutable_data_ptr(), *wp = ws->mutable_data_ptr();
        float* lp = lse ? (float*)lse->mutable_data_ptr() : nullptr;
        const int64_t qs = token_stride(*q);
        int rc;
        {
            NoLock _;
            rc = abi.paged(&c, qp, qs, op, lp, (const int*)pp, prefix_len, Hq, max_q, max_kv, (float)scale, wp, bytes, w.handle);
        }
        if (rc != 0) return nullptr;
        return tuple_of({given_or_new(a[11], o_new), lse_new.defined() ? THPVariable_Wrap(lse_new) : Py_NewRef(a[12])});
    });
}

// the addresses of the library's entry points, in the order of `abi`
PyObject* bind(PyObject*, PyObject* const* a, Py_ssize_t n) {
    if (n != 9) {
        PyErr_SetString(PyExc_TypeError, "nine addresses");
        return nullptr;
    }
    void* p[9];
    for (int i = 0; i < 9; ++i) p[i] = PyLong_AsVoidPtr(a[i]);
    if (PyErr_Occurred()) return nullptr;
    abi = {reinterpret_cast<decltype(abi.attn)>(p[0]), reinterpret_cast<decltype(abi.attn_o16)>(p[1]), reinterpret_cast<decltype(abi.softmax)>(p[2]),
           reinterpret_cast<decltype(abi.rmsnorm)>(p[3]), reinterpret_cast<decltype(abi.gemm)>(p[4]),
           reinterpret_cast<decltype(abi.residual_norm)>(p[5]), reinterpret_cast<decltype(abi.append)>(p[6]), reinterpret_cast<decltype(abi.paged)>(p[7]),
           reinterpret_cast<decltype(abi.paged_workspace)>(p[8])};
    Py_RETURN_NONE;
}

PyMethodDef methods[] = {{"bind", (PyCFunction)(void*)bind, METH_FASTCALL, nullptr},
                         {"attn_fwd", (PyCFunction)(void*)fast_attn, METH_FASTCALL, nullptr},
                         {"softmax_rows_fwd", (PyCFunction)(void*)fast_softmax, METH_FASTCALL, nullptr},
                         {"rmsnorm_fwd", (PyCFunction)(void*)fast_rmsnorm, METH_FASTCALL, nullptr},
                         {"gemm_leakyrelu_fwd", (PyCFunction)(void*)fast_gemm, METH_FASTCALL, nullptr},
                         {"residual_rmsnorm_fwd", (PyCFunction)(void*)fast_residual_norm, METH_FASTCALL, nullptr},
                         {"residual_rmsnorm_fwd_fp8", (PyCFunction)(void*)fast_residual_norm_fp8, METH_FASTCALL, nullptr},
                         {"attn_kv_append", (PyCFunction)(void*)fast_append, METH_FASTCALL, nullptr},
                         {"attn_paged_fwd", (PyCFunction)(void*)fast_paged, METH_FASTCALL, nullptr},
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_binding_fast", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__binding_fast(void) { return PyModule_Create(&module); }
