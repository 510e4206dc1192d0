// The marshalling of binding.py's smallest calls without the interpreter in between: it asks each tensor for its size, place,
// layout and address in C++ and calls the library's C function.  4096 x 4096 at M = 1 takes 4.5 us on the GPU, and asking from
// Python took longer than that.
//
// A function returns the library's status, or None for everything that is not the plain case (another type than torch.Tensor, a
// torch function mode, a tensor that is too small, on the host or not contiguous, numbers that do not fit): binding.py then goes its
// own way, with its own errors.  Nothing is kept between calls but the addresses of the library's functions.
//
// Layouts of torch, Python and qail.h are compiled in, so the module says what it was built for (`built_for`) and binding.py uses it with
// nothing else.
#define PY_SSIZE_T_CLEAN
#include <ATen/PythonTorchFunctionTLS.h>
#include <c10/hip/HIPStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include <climits>

#include "qail.h"

namespace {

decltype(&qail_w4a16_linear) g_linear = nullptr;
decltype(&qail_w4a16_linear_batch) g_linear_batch = nullptr;
decltype(&qail_w4a4_conv_batch) g_conv_batch = nullptr;
decltype(&qail_rmsnorm) g_rmsnorm = nullptr;
decltype(&qail_rmsnorm_backward) g_rmsnorm_backward = nullptr;
decltype(&qail_kv_append) g_kv_append = nullptr;
decltype(&qail_paged_attention) g_paged_attention = nullptr;
decltype(&qail_w4a16_linear_adapters_batch) g_adapters_batch = nullptr;

bool number(PyObject* o, int32_t& v) {   // an int of at least 0 that fits 32 bits
    if (!PyLong_CheckExact(o)) return false;
    int overflow = 0;
    const long long l = PyLong_AsLongLongAndOverflow(o, &overflow);
    if (overflow || l < 0 || l > INT_MAX) return false;
    v = (int32_t)l;
    return true;
}

// The address of a plain contiguous tensor on the GPU of at least `need` bytes.
template <typename T>
bool tensor(PyObject* o, int64_t need, T*& p, size_t* nbytes = nullptr) {
    if (!THPVariable_CheckExact(o)) return false;
    const at::Tensor& t = THPVariable_Unpack(o);
    if (!t.is_cuda() || !t.is_contiguous() || (int64_t)t.nbytes() < need) return false;
    p = static_cast<T*>(t.data_ptr());
    if (nbytes) *nbytes = t.nbytes();
    return true;
}

// The same of a given type, or None where `p` is NULL then; bf16 may come as 16-bit integers.
enum class Kind { bf16, fp32, int32, any };
bool is(const at::Tensor& t, Kind k) {
    const auto s = t.scalar_type();
    return k == Kind::any || (k == Kind::bf16 && (s == at::kBFloat16 || s == at::kShort)) || (k == Kind::fp32 && s == at::kFloat) || (k == Kind::int32 && s == at::kInt);
}
template <typename T>
bool typed(PyObject* o, Kind k, int64_t need, T*& p) {
    return THPVariable_CheckExact(o) && is(THPVariable_Unpack(o), k) && tensor(o, need, p);
}
template <typename T>
bool optional(PyObject* o, Kind k, int64_t need, T*& p) {
    p = nullptr;
    return o == Py_None || typed(o, k, need, p);
}
bool real(PyObject* o, float& v) {
    if (!PyFloat_CheckExact(o)) return false;
    v = (float)PyFloat_AS_DOUBLE(o);
    return true;
}
// Rows and columns of a tensor.
bool rows_of(PyObject* o, int64_t& M, int64_t& K) {
    if (!THPVariable_CheckExact(o) || THPVariable_Unpack(o).dim() != 2) return false;
    M = THPVariable_Unpack(o).size(0);
    K = THPVariable_Unpack(o).size(1);
    return M <= INT_MAX && K <= INT_MAX && M * K <= INT_MAX;
}
// bf16 [tokens, heads, dim] whose tokens may lie apart: address, stride between tokens, heads.
bool heads_of(PyObject* o, int64_t tokens, int64_t dim, const uint16_t*& p, int64_t& stride, int32_t& heads) {
    if (!THPVariable_CheckExact(o)) return false;
    const at::Tensor& t = THPVariable_Unpack(o);
    if (!t.is_cuda() || !is(t, Kind::bf16) || t.dim() != 3 || t.size(0) < tokens || t.size(2) != dim || t.stride(2) != 1 ||
        (t.stride(1) != dim && t.size(1) != 1) || t.size(1) > INT_MAX)
        return false;
    p = static_cast<const uint16_t*>(t.data_ptr());
    heads = (int32_t)t.size(1);
    stride = t.size(0) > 1 ? t.stride(0) : heads * dim;   // one token's says nothing
    return true;
}

// The array a ctypes object holds.
struct Items {
    Py_buffer view{};
    explicit Items(PyObject* o) {
        if (PyObject_GetBuffer(o, &view, PyBUF_SIMPLE) != 0) {
            PyErr_Clear();
            view.buf = nullptr;
        }
    }
    ~Items() {
        if (view.buf) PyBuffer_Release(&view);
    }
};

template <typename F>
PyObject* call(F f) {
    int status;
    Py_BEGIN_ALLOW_THREADS
    status = f();
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(status);
}

// Runs f, which returns nullptr where the call is not a plain one; whatever torch throws is left to the other way too.
template <typename F>
PyObject* plainly(F f) {
    PyObject* r = nullptr;
    try {
        if (!at::impl::torch_function_mode_enabled()) r = f();
    } catch (...) {
        PyErr_Clear();
    }
    if (r) return r;
    Py_RETURN_NONE;
}

void* stream() { return c10::hip::getCurrentHIPStream().stream(); }

// (N, K, group_size, qweight, scales, zeros, x, y, M, workspace)
PyObject* w4a16_linear(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return plainly([&]() -> PyObject* {
        int32_t N, K, g, M;
        if (n != 10 || !g_linear || !number(a[0], N) || !number(a[1], K) || !number(a[2], g) || !number(a[8], M) || g == 0) return nullptr;
        const int64_t G = K / g;
        const uint32_t *q, *z;
        const uint16_t *s, *x;
        uint16_t* y;
        void* ws = nullptr;
        size_t ws_bytes = 0;
        if (!tensor(a[3], (int64_t)N * K / 2, q) || !tensor(a[4], N * G * 2, s) || !tensor(a[5], N * ((G + 7) / 8) * 4, z) ||
            !tensor(a[6], (int64_t)M * K * 2, x) || !tensor(a[7], (int64_t)M * N * 2, y) ||
            (a[9] != Py_None && !tensor(a[9], 0, ws, &ws_bytes)))
            return nullptr;
        const qail_wdesc d = {N, K, g, QAIL_W4_ASYM_GROUP};
        void* const st = stream();
        return call([&] { return g_linear(&d, q, s, z, x, y, M, ws, ws_bytes, st); });
    });
}

// (items, count, M, workspace)
PyObject* w4a16_linear_batch(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return plainly([&]() -> PyObject* {
        int32_t count, M;
        void* ws = nullptr;
        size_t ws_bytes = 0;
        if (n != 4 || !g_linear_batch || !number(a[1], count) || !number(a[2], M) || (a[3] != Py_None && !tensor(a[3], 0, ws, &ws_bytes)))
            return nullptr;
        const Items items(a[0]);
        if (!items.view.buf) return nullptr;
        void* const st = stream();
        return call([&] { return g_linear_batch(static_cast<const qail_w4a16_item*>(items.view.buf), count, M, ws, ws_bytes, st); });
    });
}

// (items, count)
PyObject* w4a4_conv_batch(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return plainly([&]() -> PyObject* {
        int32_t count;
        if (n != 2 || !g_conv_batch || !number(a[1], count)) return nullptr;
        const Items items(a[0]);
        if (!items.view.buf) return nullptr;
        void* const st = stream();
        return call([&] { return g_conv_batch(static_cast<const qail_conv_item*>(items.view.buf), count, st); });
    });
}

// The structure of type T that a ctypes object holds.
template <typename T>
const T* held(const Items& i) { return i.view.buf && i.view.len == (Py_ssize_t)sizeof(T) ? static_cast<const T*>(i.view.buf) : nullptr; }

// (x, weight, eps, residual, residual_out, y, y_s8, y_scale)
PyObject* rmsnorm(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return plainly([&]() -> PyObject* {
        int64_t M, K;
        float eps;
        const uint16_t *x, *weight, *residual;
        uint16_t *h, *y;
        uint32_t* codes;
        float* scale;
        if (n != 8 || !g_rmsnorm || !rows_of(a[0], M, K) || !real(a[2], eps) || !typed(a[0], Kind::bf16, M * K * 2, x) || !typed(a[1], Kind::bf16, K * 2, weight) ||
            !optional(a[3], Kind::bf16, M * K * 2, residual) || !optional(a[4], Kind::bf16, M * K * 2, h) || !optional(a[5], Kind::bf16, M * K * 2, y) ||
            !optional(a[6], Kind::any, M * K, codes) || !optional(a[7], Kind::fp32, M * 4, scale))
            return nullptr;
        void* const st = stream();
        return call([&] { return g_rmsnorm(x, residual, weight, eps, (int32_t)M, (int32_t)K, h, y, codes, scale, st); });
    });
}

// (h, weight, eps, dy, dx, dweight, workspace, dres)
PyObject* rmsnorm_backward(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return plainly([&]() -> PyObject* {
        int64_t M, K;
        float eps;
        const uint16_t *h, *weight, *dy, *dres;
        uint16_t* dx;
        float* dw;
        void* ws;
        size_t ws_bytes = 0;
        if (n != 8 || !g_rmsnorm_backward || !rows_of(a[0], M, K) || !real(a[2], eps) || !typed(a[0], Kind::bf16, M * K * 2, h) ||
            !typed(a[1], Kind::bf16, K * 2, weight) || !typed(a[3], Kind::bf16, M * K * 2, dy) || !typed(a[4], Kind::bf16, M * K * 2, dx) ||
            !typed(a[5], Kind::fp32, K * 4, dw) || !tensor(a[6], 0, ws, &ws_bytes) || !optional(a[7], Kind::bf16, M * K * 2, dres))
            return nullptr;
        void* const st = stream();
        return call([&] { return g_rmsnorm_backward(h, weight, eps, dy, dres, (int32_t)M, (int32_t)K, dx, dw, ws, ws_bytes, st); });
    });
}

// (cache, requests, k, v, q, q_out, cos, sin, errors)
PyObject* kv_append(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return plainly([&]() -> PyObject* {
        if (n != 9 || !g_kv_append) return nullptr;
        const Items ci(a[0]), bi(a[1]);
        const auto* c = held<qail_kv_cache>(ci);
        const auto* b = held<qail_requests>(bi);
        const uint16_t *k, *v, *q = nullptr;
        uint16_t* out;
        const float *cos, *sin;
        uint32_t* errors;
        int64_t ks, vs, qs = 0, positions = 0;
        int32_t kh, vh, qh = 0;
        if (!c || !b || !heads_of(a[2], b->tokens, c->head_dim, k, ks, kh) || !heads_of(a[3], b->tokens, c->head_dim, v, vs, vh) || kh != c->heads || vh != c->heads ||
            (a[4] != Py_None && !heads_of(a[4], b->tokens, c->head_dim, q, qs, qh)) || !optional(a[5], Kind::bf16, (int64_t)b->tokens * qh * c->head_dim * 2, out))
            return nullptr;
        if (a[6] != Py_None) {
            if (!THPVariable_CheckExact(a[6]) || THPVariable_Unpack(a[6]).dim() < 1) return nullptr;
            positions = THPVariable_Unpack(a[6]).size(0);
            if (positions > INT_MAX) return nullptr;
        }
        if (!optional(a[6], Kind::fp32, positions * c->head_dim * 2, cos) || !optional(a[7], Kind::fp32, positions * c->head_dim * 2, sin) ||
            !optional(a[8], Kind::int32, 4, errors))
            return nullptr;
        void* const st = stream();
        return call([&] { return g_kv_append(c, b, k, ks, v, vs, q, qs, qh, out, cos, sin, (int32_t)positions, errors, st); });
    });
}

// (cache, requests, q, out, scale, workspace, errors)
PyObject* paged_attention(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return plainly([&]() -> PyObject* {
        if (n != 7 || !g_paged_attention) return nullptr;
        const Items ci(a[0]), bi(a[1]);
        const auto* c = held<qail_kv_cache>(ci);
        const auto* b = held<qail_requests>(bi);
        const uint16_t* q;
        uint16_t* out;
        uint32_t* errors;
        void* ws = nullptr;
        size_t ws_bytes = 0;
        int64_t qs;
        int32_t qh;
        float scale;
        if (!c || !b || !heads_of(a[2], b->tokens, c->head_dim, q, qs, qh) || !typed(a[3], Kind::bf16, (int64_t)b->tokens * qh * c->head_dim * 2, out) ||
            !real(a[4], scale) || (a[5] != Py_None && !tensor(a[5], 0, ws, &ws_bytes)) || !optional(a[6], Kind::int32, 4, errors))
            return nullptr;
        void* const st = stream();
        return call([&] { return g_paged_attention(c, b, q, qs, qh, scale, out, errors, ws, ws_bytes, st); });
    });
}

// (items, adapters, row_adapter, count, M, workspace)
PyObject* adapters_batch(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return plainly([&]() -> PyObject* {
        int32_t count, M;
        const int32_t* rows;
        void* ws;
        size_t ws_bytes = 0;
        if (n != 6 || !g_adapters_batch || !number(a[3], count) || !number(a[4], M) || !typed(a[2], Kind::int32, (int64_t)M * 4, rows) || !tensor(a[5], 0, ws, &ws_bytes))
            return nullptr;
        const Items items(a[0]), adapters(a[1]);
        if (!items.view.buf || !adapters.view.buf || items.view.len < (Py_ssize_t)(count * sizeof(qail_w4a16_item)) ||
            adapters.view.len < (Py_ssize_t)(count * sizeof(qail_adapters)))
            return nullptr;
        void* const st = stream();
        return call([&] {
            return g_adapters_batch(static_cast<const qail_w4a16_item*>(items.view.buf), static_cast<const qail_adapters*>(adapters.view.buf), rows, count, M, ws, ws_bytes, st);
        });
    });
}

// Addresses of the five functions of serving, in the order above.
PyObject* use_serving(PyObject*, PyObject* args) {
    unsigned long long f[5];
    if (!PyArg_ParseTuple(args, "KKKKK", &f[0], &f[1], &f[2], &f[3], &f[4])) return nullptr;
    g_rmsnorm = reinterpret_cast<decltype(g_rmsnorm)>(f[0]);
    g_rmsnorm_backward = reinterpret_cast<decltype(g_rmsnorm_backward)>(f[1]);
    g_kv_append = reinterpret_cast<decltype(g_kv_append)>(f[2]);
    g_paged_attention = reinterpret_cast<decltype(g_paged_attention)>(f[3]);
    g_adapters_batch = reinterpret_cast<decltype(g_adapters_batch)>(f[4]);
    Py_RETURN_NONE;
}

// Addresses of qail_w4a16_linear, qail_w4a16_linear_batch and qail_w4a4_conv_batch.
PyObject* use(PyObject*, PyObject* args) {
    unsigned long long l, b, c;
    if (!PyArg_ParseTuple(args, "KKK", &l, &b, &c)) return nullptr;
    g_linear = reinterpret_cast<decltype(g_linear)>(l);
    g_linear_batch = reinterpret_cast<decltype(g_linear_batch)>(b);
    g_conv_batch = reinterpret_cast<decltype(g_conv_batch)>(c);
    Py_RETURN_NONE;
}

PyMethodDef methods[] = {
    {"use", use, METH_VARARGS, nullptr},
    {"use_serving", use_serving, METH_VARARGS, nullptr},
    {"rmsnorm", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(rmsnorm)), METH_FASTCALL, nullptr},
    {"rmsnorm_backward", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(rmsnorm_backward)), METH_FASTCALL, nullptr},
    {"kv_append", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(kv_append)), METH_FASTCALL, nullptr},
    {"paged_attention", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(paged_attention)), METH_FASTCALL, nullptr},
    {"adapters_batch", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(adapters_batch)), METH_FASTCALL, nullptr},
    {"w4a16_linear", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(w4a16_linear)), METH_FASTCALL, nullptr},
    {"w4a16_linear_batch", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(w4a16_linear_batch)), METH_FASTCALL, nullptr},
    {"w4a4_conv_batch", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(w4a4_conv_batch)), METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr},
};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_marshal", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__marshal() {
    PyObject* m = PyModule_Create(&module);
    PyObject* built_for = m ? Py_BuildValue("(lsnnnnnn)", (long)(PY_VERSION_HEX >> 16), QAIL_TORCH, (Py_ssize_t)sizeof(qail_wdesc),
                                            (Py_ssize_t)sizeof(qail_w4a16_item), (Py_ssize_t)sizeof(qail_conv_item), (Py_ssize_t)sizeof(qail_kv_cache),
                                            (Py_ssize_t)sizeof(qail_requests), (Py_ssize_t)sizeof(qail_adapters))
                            : nullptr;
    if (!built_for || PyModule_AddObject(m, "built_for", built_for) < 0) {   // (takes the reference where it succeeds)
        Py_XDECREF(built_for);
        Py_XDECREF(m);
        return nullptr;
    }
    return m;
}
