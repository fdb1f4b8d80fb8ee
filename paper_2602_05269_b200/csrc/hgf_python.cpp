// The marshalling of hgf.linear_forward and of the cache calls in native code: tensors to addresses, the current stream, the call.  The smallest
// layers take 4 us on the GPU, and a decode loop makes such calls one after the other: 512 -> 512, M = 4 took 10.5 us a call through ctypes, which
// the host spent on arguments, and takes 4.5 us now (one B200, calls back to back).  A cache call took the host 10 us.
#include <torch/csrc/autograd/python_variable.h>

#include <ATen/cuda/CUDAContext.h>

#include "../../include/hgf.h"

namespace {

decltype(&hgf_linear_forward) g_forward = nullptr;
decltype(&hgf_linear_forward_ln) g_forward_ln = nullptr;

// A tensor that is exactly one (or a Parameter); anything else answers through its own methods.
const at::Tensor *plain_tensor(PyObject *o) { return THPVariable_CheckExact(o) ? &THPVariable_Unpack(o) : nullptr; }

// A Python int, nothing that turns into one (TypeError: the caller goes through ctypes then, which takes ints alone, too).
bool integer(PyObject *o, unsigned long long *out) {
    if (!PyLong_Check(o)) {
        PyErr_SetString(PyExc_TypeError, "int expected");
        return false;
    }
    *out = PyLong_AsUnsignedLongLongMask(o);
    return true;
}
bool method_value(PyObject *o, const char *name, unsigned long long *out) {
    PyObject *v = PyObject_CallMethod(o, name, nullptr);
    if (!v) return false;
    const bool ok = integer(v, out);
    Py_DECREF(v);
    return ok;
}
bool address(PyObject *o, void **out) {
    *out = nullptr;
    if (o == Py_None) return true;
    if (const at::Tensor *t = plain_tensor(o)) {
        *out = t->data_ptr();
        return true;
    }
    unsigned long long v = 0;
    if (!method_value(o, "data_ptr", &v)) return false;
    *out = reinterpret_cast<void *>(v);
    return true;
}
bool elements(PyObject *o, size_t *out) {
    if (const at::Tensor *t = plain_tensor(o)) {
        *out = (size_t)t->numel();
        return true;
    }
    unsigned long long v = 0;
    if (!method_value(o, "numel", &v)) return false;
    *out = (size_t)v;
    return true;
}
bool rows(PyObject *o, int64_t *out) {  // shape[0]
    const at::Tensor *t = plain_tensor(o);
    if (t && t->dim() > 0) {
        *out = t->size(0);
        return true;
    }
    PyObject *shape = PyObject_GetAttrString(o, "shape");
    PyObject *first = shape ? PySequence_GetItem(shape, 0) : nullptr;
    Py_XDECREF(shape);
    if (!first) return false;
    unsigned long long v = 0;
    const bool ok = integer(first, &v);
    *out = (int64_t)v;
    Py_DECREF(first);
    return ok;
}
bool integer(PyObject *o, int64_t *out) {
    unsigned long long v = 0;
    const bool ok = integer(o, &v);
    *out = (int64_t)v;
    return ok;
}

// linear_forward(x, packed, gamma, d_in, d_out, At, Bt, gate, y, workspace, flags, stream, ln_weight, ln_bias, eps, gate_group) -> status
PyObject *linear_forward(PyObject *, PyObject *const *a, Py_ssize_t n) try {
    if (n != 16) {
        PyErr_SetString(PyExc_TypeError, "linear_forward takes 16 arguments");
        return nullptr;
    }
    void *x, *packed, *At, *Bt, *gate, *y, *workspace, *ln_weight, *ln_bias, *stream;
    int64_t M, d_in, d_out, r = 0, flags, gate_group = 1;
    size_t workspace_bytes = 0;
    if (!rows(a[0], &M) || !address(a[0], &x) || !address(a[1], &packed) || !integer(a[3], &d_in) || !integer(a[4], &d_out) ||
        !address(a[5], &At) || !address(a[6], &Bt) || !address(a[7], &gate) || !address(a[8], &y) || !address(a[9], &workspace) ||
        !elements(a[9], &workspace_bytes) || !integer(a[10], &flags))
        return nullptr;
    if (a[5] != Py_None && !rows(a[5], &r)) return nullptr;
    const float gamma = (float)PyFloat_AsDouble(a[2]);
    if (PyErr_Occurred()) return nullptr;
    if (a[11] == Py_None) {
        stream = at::cuda::getCurrentCUDAStream().stream();
    } else {
        PyObject *s = PyObject_GetAttrString(a[11], "cuda_stream");
        if (!s) return nullptr;
        unsigned long long v = 0;
        const bool ok = integer(s, &v);
        Py_DECREF(s);
        if (!ok) return nullptr;
        stream = reinterpret_cast<void *>(v);
    }
    hgf_front_end fe = {};
    const bool front_end = a[12] != Py_None || a[15] != Py_None;
    if (front_end) {
        if (!address(a[12], &ln_weight) || !address(a[13], &ln_bias)) return nullptr;
        fe.ln_weight = (const float *)ln_weight;
        fe.ln_bias = (const float *)ln_bias;
        fe.eps = (float)PyFloat_AsDouble(a[14]);
        if (PyErr_Occurred() || (a[15] != Py_None && !integer(a[15], &gate_group))) return nullptr;
        fe.gate_group = gate_group ? gate_group : 1;
    }
    hgf_status st;
    Py_BEGIN_ALLOW_THREADS
    st = front_end ? g_forward_ln(x, M, packed, gamma, d_in, d_out, At, Bt, (int32_t)r, (const float *)gate, y, workspace, workspace_bytes, nullptr, &fe, (uint32_t)flags, stream)
                   : g_forward(x, M, packed, gamma, d_in, d_out, At, Bt, (int32_t)r, (const float *)gate, y, workspace, workspace_bytes, nullptr, (uint32_t)flags, stream);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong((long)st);
} catch (const std::exception &e) {  // (of torch: no device, a tensor without storage)
    PyErr_SetString(PyExc_RuntimeError, e.what());
    return nullptr;
}

// ---- cache calls ----------------------------------------------------------------------------------------------------------------
// Each takes the address of an hgf_cache, its device's number, and the arguments of the function of the same name in hgf.py, and returns the status;
// -1 where an argument is not the plain, dense tensor on that device that the call takes, with nothing called (hgf.py then says what is wrong).
decltype(&hgf_cache_reserve) g_reserve = nullptr;
decltype(&hgf_cache_append) g_append = nullptr;
decltype(&hgf_cache_read) g_read = nullptr;
decltype(&hgf_cache_fork) g_fork = nullptr;
decltype(&hgf_cache_free) g_free = nullptr;
decltype(&hgf_diff_attention_cached) g_attend = nullptr;

// A call on tensors of the current device: its stream, and whether all that it has been given is what it takes.
struct DeviceCall {
    int64_t device = -1;
    void *stream = nullptr;
    bool ok = true;

    void begin(PyObject *stream_) {
        ok = ok && device >= 0 && device == (int64_t)at::cuda::current_device();
        if (!ok) return;
        unsigned long long v = 0;
        if (stream_ == Py_None) {
            stream = at::cuda::getCurrentCUDAStream().stream();
        } else {
            PyObject *s = PyObject_GetAttrString(stream_, "cuda_stream");
            ok = s && integer(s, &v);
            Py_XDECREF(s);
            stream = reinterpret_cast<void *>(v);
        }
    }
    // The device of the first tensor that is one.
    DeviceCall &of(PyObject *o) {
        const at::Tensor *t = plain_tensor(o);
        if (device < 0 && t && t->is_cuda()) device = t->device().index();
        return *this;
    }
    const at::Tensor *tensor(PyObject *o, at::ScalarType type) {
        const at::Tensor *t = plain_tensor(o);
        ok = ok && t && t->scalar_type() == type && t->is_cuda() && t->device().index() == device && t->is_contiguous();
        return ok ? t : nullptr;
    }
    const int32_t *list(PyObject *o, int64_t n) {
        const at::Tensor *t = tensor(o, at::kInt);
        ok = ok && t->dim() == 1 && t->size(0) == n;
        return ok ? static_cast<const int32_t *>(t->data_ptr()) : nullptr;
    }
    int64_t count(PyObject *o) {
        const at::Tensor *t = plain_tensor(o);
        ok = ok && t && t->dim() == 1;
        return ok ? t->size(0) : 0;
    }
    void *matrix(PyObject *o, at::ScalarType type, int64_t rows, int64_t cols) {
        const at::Tensor *t = tensor(o, type);
        ok = ok && t->dim() == 2 && t->size(0) == rows && t->size(1) == cols;
        return ok ? t->data_ptr() : nullptr;
    }
    int64_t height(PyObject *o) {
        const at::Tensor *t = plain_tensor(o);
        ok = ok && t && t->dim() == 2;
        return ok ? t->size(0) : 0;
    }
    int64_t cols(PyObject *o) { return height(o) || ok ? plain_tensor(o)->size(1) : 0; }
    void *vector(PyObject *o, at::ScalarType type, int64_t n) {
        const at::Tensor *t = tensor(o, type);
        ok = ok && t->dim() == 1 && t->size(0) == n;
        return ok ? t->data_ptr() : nullptr;
    }
    // (None: a null pointer)
    void *matrix_or_none(PyObject *o, at::ScalarType type, int64_t rows, int64_t n) { return o == Py_None ? nullptr : matrix(o, type, rows, n); }
    void *vector_or_none(PyObject *o, at::ScalarType type, int64_t n) { return o == Py_None ? nullptr : vector(o, type, n); }
    double number(PyObject *o) {
        const double v = PyFloat_AsDouble(o);
        ok = ok && !(v == -1.0 && PyErr_Occurred());
        return v;
    }
    int64_t whole(PyObject *o) {
        int64_t v = 0;
        ok = ok && integer(o, &v);
        return v;
    }
};
struct CacheCall : DeviceCall {
    const hgf_cache *cache;

    CacheCall(PyObject *at, PyObject *dev, PyObject *stream_) {
        unsigned long long v = 0, d = 0;
        ok = integer(at, &v) && integer(dev, &d);  // (a cache in host memory has -1)
        cache = reinterpret_cast<const hgf_cache *>(v);
        device = (int64_t)d;
        begin(stream_);
    }
};
PyObject *given_back() { return PyErr_Occurred() ? nullptr : PyLong_FromLong(-1); }
template <class F>
PyObject *called(F f) {
    hgf_status st;
    Py_BEGIN_ALLOW_THREADS
    st = f();
    Py_END_ALLOW_THREADS
    return PyLong_FromLong((long)st);
}
template <class F>
PyObject *guarded(Py_ssize_t n, Py_ssize_t want, F f) try {
    if (n != want) {
        PyErr_SetString(PyExc_TypeError, "wrong number of arguments");
        return nullptr;
    }
    return f();
} catch (const std::exception &e) {
    PyErr_SetString(PyExc_RuntimeError, e.what());
    return nullptr;
}

// (cache, device, slots, tokens, granted, stream)
PyObject *cache_reserve(PyObject *, PyObject *const *a, Py_ssize_t n_) {
    return guarded(n_, 6, [&]() -> PyObject * {
        CacheCall c(a[0], a[1], a[5]);
        const int64_t n = c.count(a[2]);
        const int32_t *slots = c.list(a[2], n), *tokens = c.list(a[3], n), *granted = c.list(a[4], n);
        if (!c.ok) return given_back();
        return called([&] { return g_reserve(c.cache, slots, tokens, n, const_cast<int32_t *>(granted), c.stream); });
    });
}
// (cache, device, k, v, slots, starts, done, stream)
PyObject *cache_append(PyObject *, PyObject *const *a, Py_ssize_t n_) {
    return guarded(n_, 8, [&]() -> PyObject * {
        CacheCall c(a[0], a[1], a[7]);
        const int64_t n = c.count(a[4]), rows = c.height(a[2]), width = c.ok ? (int64_t)c.cache->n_heads * c.cache->head_dim : 0;
        const void *k = c.matrix(a[2], at::kBFloat16, rows, 2 * width), *v = c.matrix(a[3], at::kBFloat16, rows, width);
        const int32_t *slots = c.list(a[4], n), *starts = c.list(a[5], n + 1), *done = c.list(a[6], n);
        if (!c.ok) return given_back();
        return called([&] { return g_append(c.cache, k, v, rows, slots, starts, n, const_cast<int32_t *>(done), c.stream); });
    });
}
// (cache, device, slots, first, starts, k, v, stream): the type of k and v says which
PyObject *cache_read(PyObject *, PyObject *const *a, Py_ssize_t n_) {
    return guarded(n_, 8, [&]() -> PyObject * {
        CacheCall c(a[0], a[1], a[7]);
        const int64_t n = c.count(a[2]), rows = c.height(a[5]), width = c.ok ? (int64_t)c.cache->n_heads * c.cache->head_dim : 0;
        const at::ScalarType type = c.ok && plain_tensor(a[5])->scalar_type() == at::kBFloat16 ? at::kBFloat16 : at::kFloat;
        void *k = c.matrix(a[5], type, rows, 2 * width), *v = c.matrix(a[6], type, rows, width);
        const int32_t *slots = c.list(a[2], n), *first = c.list(a[3], n), *starts = c.list(a[4], n + 1);
        if (!c.ok) return given_back();
        return called([&] { return g_read(c.cache, slots, first, starts, n, rows, k, v, type == at::kBFloat16 ? HGF_FLAG_OUT_BF16 : 0u, c.stream); });
    });
}
// (cache, device, src, dst, done, stream)
PyObject *cache_fork(PyObject *, PyObject *const *a, Py_ssize_t n_) {
    return guarded(n_, 6, [&]() -> PyObject * {
        CacheCall c(a[0], a[1], a[5]);
        const int64_t n = c.count(a[2]);
        const int32_t *src = c.list(a[2], n), *dst = c.list(a[3], n), *done = c.list(a[4], n);
        if (!c.ok) return given_back();
        return called([&] { return g_fork(c.cache, src, dst, n, const_cast<int32_t *>(done), c.stream); });
    });
}
// (cache, device, slots, stream)
PyObject *cache_free(PyObject *, PyObject *const *a, Py_ssize_t n_) {
    return guarded(n_, 4, [&]() -> PyObject * {
        CacheCall c(a[0], a[1], a[3]);
        const int64_t n = c.count(a[2]);
        const int32_t *slots = c.list(a[2], n);
        if (!c.ok) return given_back();
        return called([&] { return g_free(c.cache, slots, n, c.stream); });
    });
}
// (cache, device, q, slots, starts, lambda, out_scale, out, workspace, flags, stream)
PyObject *diff_attention_cached(PyObject *, PyObject *const *a, Py_ssize_t n_) {
    return guarded(n_, 11, [&]() -> PyObject * {
        CacheCall c(a[0], a[1], a[10]);
        const int64_t n = c.count(a[3]), rows = c.height(a[2]);
        int64_t flags = 0;
        if (!integer(a[9], &flags)) return nullptr;
        const double lambda = PyFloat_AsDouble(a[5]), out_scale = PyFloat_AsDouble(a[6]);
        if (PyErr_Occurred()) return nullptr;
        const at::Tensor *q = c.tensor(a[2], at::kBFloat16);
        if (!c.ok) return given_back();
        const int64_t pair = 2 * (int64_t)c.cache->head_dim, heads = q->size(1) / pair;
        c.ok = q->size(1) == heads * pair;
        void *out = c.matrix(a[7], flags & HGF_FLAG_OUT_BF16 ? at::kBFloat16 : at::kFloat, rows, heads * pair / 2);
        const at::Tensor *workspace = c.tensor(a[8], at::kByte);
        const int32_t *slots = c.list(a[3], n), *starts = c.list(a[4], n + 1);
        if (!c.ok || heads > INT32_MAX) return given_back();
        return called([&] {
            return g_attend(c.cache, q->data_ptr(), rows, (int32_t)heads, slots, starts, n, (float)lambda, (float)out_scale, out, workspace->data_ptr(),
                            (size_t)workspace->numel(), (uint32_t)flags, c.stream);
        });
    });
}
// bind_cache(addresses of the six calls, in the order above)
PyObject *bind_cache(PyObject *, PyObject *args) {
    unsigned long long f[6];
    if (!PyArg_ParseTuple(args, "KKKKKK", f, f + 1, f + 2, f + 3, f + 4, f + 5)) return nullptr;
    g_reserve = reinterpret_cast<decltype(g_reserve)>(f[0]);
    g_append = reinterpret_cast<decltype(g_append)>(f[1]);
    g_read = reinterpret_cast<decltype(g_read)>(f[2]);
    g_fork = reinterpret_cast<decltype(g_fork)>(f[3]);
    g_free = reinterpret_cast<decltype(g_free)>(f[4]);
    g_attend = reinterpret_cast<decltype(g_attend)>(f[5]);
    Py_RETURN_NONE;
}

// ---- training calls -----------------------------------------------------------------------------------------------------------
// As the cache calls: the arguments of the function of the same name in hgf.py, every tensor made already; -1 where one is not what the call takes.
decltype(&hgf_diff_attention_forward_train) g_attention = nullptr;
decltype(&hgf_diff_attention_backward) g_attention_backward = nullptr;
decltype(&hgf_qk_norm_rotate) g_rotate = nullptr;
decltype(&hgf_qk_norm_rotate_backward) g_rotate_backward = nullptr;
decltype(&hgf_clip_grad_norm) g_clip = nullptr;

struct AttentionCall : DeviceCall {
    int64_t B, L, h, dh, width = 0, rows = 0;
    double lambda, scale;
    const void *q, *k, *v;
    const float *streams, *lse;
    // q, k, v, then at n: B, L, n_heads, head_dim, lambda, out_scale
    AttentionCall(PyObject *const *a, int n, PyObject *streams_, PyObject *lse_, PyObject *stream_) {
        of(a[0]);
        begin(stream_);
        B = whole(a[n]), L = whole(a[n + 1]), h = whole(a[n + 2]), dh = whole(a[n + 3]);
        lambda = number(a[n + 4]), scale = number(a[n + 5]);
        ok = ok && B > 0 && L > 0 && h > 0 && dh > 0 && B < (1 << 24) && L < (1ll << 32) && h < (1 << 24) && dh < (1 << 12);
        if (!ok) return;
        rows = B * L, width = h * dh;
        q = matrix(a[0], at::kBFloat16, rows, 2 * width), k = matrix(a[1], at::kBFloat16, rows, 2 * width), v = matrix(a[2], at::kBFloat16, rows, width);
        streams = static_cast<const float *>(matrix(streams_, at::kFloat, rows, 2 * width));
        const at::Tensor *t = tensor(lse_, at::kFloat);
        ok = ok && t->dim() == 4 && t->size(0) == B && t->size(1) == h && t->size(2) == 2 && t->size(3) == L;
        lse = ok ? static_cast<const float *>(t->data_ptr()) : nullptr;
    }
};
// (q, k, v, B, L, n_heads, head_dim, lambda, out_scale, out, streams, lse, flags, stream)
PyObject *diff_attention_forward_train(PyObject *, PyObject *const *a, Py_ssize_t n_) {
    return guarded(n_, 14, [&]() -> PyObject * {
        AttentionCall c(a, 3, a[10], a[11], a[13]);
        const int64_t flags = c.whole(a[12]);
        void *out = c.matrix(a[9], flags & HGF_FLAG_OUT_BF16 ? at::kBFloat16 : at::kFloat, c.rows, c.width);
        if (!c.ok) return given_back();
        return called([&] {
            return g_attention(c.q, c.k, c.v, c.B, c.L, (int32_t)c.h, (int32_t)c.dh, (float)c.lambda, (float)c.scale, out, const_cast<float *>(c.streams),
                               const_cast<float *>(c.lse), (uint32_t)flags, c.stream);
        });
    });
}
// (q, k, v, dout, streams, lse, B, L, n_heads, head_dim, lambda, out_scale, dq, dk, dv, dlambda, workspace, stream)
PyObject *diff_attention_backward(PyObject *, PyObject *const *a, Py_ssize_t n_) {
    return guarded(n_, 18, [&]() -> PyObject * {
        AttentionCall c(a, 6, a[4], a[5], a[17]);
        const void *dout = c.matrix(a[3], at::kBFloat16, c.rows, c.width);
        hgf_attention_grads g = {};
        g.dq = c.matrix_or_none(a[12], at::kBFloat16, c.rows, 2 * c.width);
        g.dk = c.matrix_or_none(a[13], at::kBFloat16, c.rows, 2 * c.width);
        g.dv = c.matrix_or_none(a[14], at::kBFloat16, c.rows, c.width);
        g.dlambda = static_cast<float *>(c.vector_or_none(a[15], at::kFloat, 1));
        const at::Tensor *workspace = c.tensor(a[16], at::kByte);
        if (!c.ok) return given_back();
        return called([&] {
            return g_attention_backward(c.q, c.k, c.v, dout, c.streams, c.lse, c.B, c.L, (int32_t)c.h, (int32_t)c.dh, (float)c.lambda, (float)c.scale, &g,
                                        workspace->data_ptr(), (size_t)workspace->numel(), 0u, c.stream);
        });
    });
}

struct RotateCall : DeviceCall {
    int64_t rows = 0, dh, rot, flags, wide_q = 0, wide_k = 0;
    const void *q = nullptr, *k = nullptr;
    const int32_t *pos = nullptr;
    const float *wq = nullptr, *wk = nullptr;
    double eps, base;
    // q, k, positions, head_dim, wq, wk, eps, base, rotary_dim, flags
    RotateCall(PyObject *const *a, PyObject *stream_) {
        of(a[0]).of(a[1]);
        begin(stream_);
        dh = whole(a[3]), eps = number(a[6]), base = number(a[7]), rot = whole(a[8]), flags = whole(a[9]);
        ok = ok && dh > 0 && dh < (1 << 12) && rot >= 0 && rot <= dh;
        if (!ok) return;
        PyObject *some = a[0] != Py_None ? a[0] : a[1];
        rows = height(some);
        if (a[0] != Py_None) wide_q = cols(a[0]);
        if (a[1] != Py_None) wide_k = cols(a[1]);
        ok = ok && wide_q % dh == 0 && wide_k % dh == 0 && (wide_q | wide_k) < (1ll << 31);
        q = matrix_or_none(a[0], at::kBFloat16, rows, wide_q), k = matrix_or_none(a[1], at::kBFloat16, rows, wide_k);
        pos = list(a[2], rows);
        wq = static_cast<const float *>(vector_or_none(a[4], at::kFloat, dh)), wk = static_cast<const float *>(vector_or_none(a[5], at::kFloat, dh));
    }
};
// (q, k, positions, head_dim, wq, wk, eps, base, rotary_dim, flags, q_out, k_out, stream)
PyObject *qk_norm_rotate(PyObject *, PyObject *const *a, Py_ssize_t n_) {
    return guarded(n_, 13, [&]() -> PyObject * {
        RotateCall c(a, a[12]);
        void *qo = c.matrix_or_none(a[10], at::kBFloat16, c.rows, c.wide_q), *ko = c.matrix_or_none(a[11], at::kBFloat16, c.rows, c.wide_k);
        if (!c.ok || !qo != !c.q || !ko != !c.k) return given_back();
        return called([&] {
            return g_rotate(c.q, c.k, c.rows, (int32_t)(c.wide_q / c.dh), (int32_t)(c.wide_k / c.dh), (int32_t)c.dh, c.pos, c.wq, c.wk, (float)c.eps, c.base,
                            (int32_t)c.rot, qo, ko, (uint32_t)c.flags, c.stream);
        });
    });
}
// (q, k, positions, head_dim, wq, wk, eps, base, rotary_dim, flags, dq_out, dk_out, dq, dk, dwq, dwk, workspace, stream)
PyObject *qk_norm_rotate_backward(PyObject *, PyObject *const *a, Py_ssize_t n_) {
    return guarded(n_, 18, [&]() -> PyObject * {
        RotateCall c(a, a[17]);
        const void *gq = c.matrix_or_none(a[10], at::kBFloat16, c.rows, c.wide_q), *gk = c.matrix_or_none(a[11], at::kBFloat16, c.rows, c.wide_k);
        hgf_rotate_grads g = {};
        g.dq = c.matrix_or_none(a[12], at::kBFloat16, c.rows, c.wide_q);
        g.dk = c.matrix_or_none(a[13], at::kBFloat16, c.rows, c.wide_k);
        g.dwq = static_cast<float *>(c.vector_or_none(a[14], at::kFloat, c.dh));
        g.dwk = static_cast<float *>(c.vector_or_none(a[15], at::kFloat, c.dh));
        const at::Tensor *workspace = c.tensor(a[16], at::kByte);
        if (!c.ok || !gq != !c.q || !gk != !c.k) return given_back();
        return called([&] {
            return g_rotate_backward(c.q, c.k, c.rows, (int32_t)(c.wide_q / c.dh), (int32_t)(c.wide_k / c.dh), (int32_t)c.dh, c.pos, c.wq, c.wk, (float)c.eps, c.base,
                                     (int32_t)c.rot, gq, gk, &g, workspace->data_ptr(), (size_t)workspace->numel(), (uint32_t)c.flags, c.stream);
        });
    });
}
// (handle, device, max_norm, norm, stream)
PyObject *clip_grad_norm(PyObject *, PyObject *const *a, Py_ssize_t n_) {
    return guarded(n_, 5, [&]() -> PyObject * {
        DeviceCall c;
        unsigned long long handle = 0;
        if (!integer(a[0], &handle) || !integer(a[1], &c.device)) return nullptr;
        c.begin(a[4]);
        const double max_norm = c.number(a[2]);
        void *norm = c.vector(a[3], at::kFloat, 1);
        if (!c.ok) return given_back();
        return called([&] { return g_clip(reinterpret_cast<hgf_grad_list *>(handle), (float)max_norm, static_cast<float *>(norm), c.stream); });
    });
}
// bind_train(addresses of the five calls, in the order above)
PyObject *bind_train(PyObject *, PyObject *args) {
    unsigned long long f[5];
    if (!PyArg_ParseTuple(args, "KKKKK", f, f + 1, f + 2, f + 3, f + 4)) return nullptr;
    g_attention = reinterpret_cast<decltype(g_attention)>(f[0]);
    g_attention_backward = reinterpret_cast<decltype(g_attention_backward)>(f[1]);
    g_rotate = reinterpret_cast<decltype(g_rotate)>(f[2]);
    g_rotate_backward = reinterpret_cast<decltype(g_rotate_backward)>(f[3]);
    g_clip = reinterpret_cast<decltype(g_clip)>(f[4]);
    Py_RETURN_NONE;
}

// bind(address of hgf_linear_forward, address of hgf_linear_forward_ln): in the library that hgf.lib() has loaded
PyObject *bind(PyObject *, PyObject *args) {
    unsigned long long forward, forward_ln;
    if (!PyArg_ParseTuple(args, "KK", &forward, &forward_ln)) return nullptr;
    g_forward = reinterpret_cast<decltype(g_forward)>(forward);
    g_forward_ln = reinterpret_cast<decltype(g_forward_ln)>(forward_ln);
    Py_RETURN_NONE;
}

PyMethodDef methods[] = {{"linear_forward", reinterpret_cast<PyCFunction>(reinterpret_cast<void *>(linear_forward)), METH_FASTCALL, nullptr},
                         {"bind", bind, METH_VARARGS, nullptr},
#define HGF_CACHE_METHOD(name) {#name, reinterpret_cast<PyCFunction>(reinterpret_cast<void *>(name)), METH_FASTCALL, nullptr}
                         HGF_CACHE_METHOD(cache_reserve), HGF_CACHE_METHOD(cache_append), HGF_CACHE_METHOD(cache_read), HGF_CACHE_METHOD(cache_fork),
                         HGF_CACHE_METHOD(cache_free), HGF_CACHE_METHOD(diff_attention_cached),
                         {"bind_cache", bind_cache, METH_VARARGS, nullptr},
                         HGF_CACHE_METHOD(diff_attention_forward_train), HGF_CACHE_METHOD(diff_attention_backward), HGF_CACHE_METHOD(qk_norm_rotate),
                         HGF_CACHE_METHOD(qk_norm_rotate_backward), HGF_CACHE_METHOD(clip_grad_norm),
                         {"bind_train", bind_train, METH_VARARGS, nullptr},
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_hgf_python", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__hgf_python() { return PyModule_Create(&module); }
