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

struct CacheCall {
    const hgf_cache *cache;
    int64_t device;
    void *stream = nullptr;
    bool ok = true;

    CacheCall(PyObject *at, PyObject *dev, PyObject *stream_) {
        unsigned long long v = 0, d = 0;
        ok = integer(at, &v) && integer(dev, &d);  // (a cache in host memory has -1)
        cache = reinterpret_cast<const hgf_cache *>(v);
        device = (int64_t)d;
        ok = ok && device >= 0 && device == (int64_t)at::cuda::current_device();
        if (!ok) return;
        if (stream_ == Py_None) {
            stream = at::cuda::getCurrentCUDAStream().stream();
        } else {
            PyObject *s = PyObject_GetAttrString(stream_, "cuda_stream");
            ok = s && integer(s, &v);
            Py_XDECREF(s);
            stream = reinterpret_cast<void *>(v);
        }
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
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_hgf_python", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__hgf_python() { return PyModule_Create(&module); }
