// The host side of a product call from Python: argument checks, the output tensor, the current stream and the call into the C
// ABI, without a Python-level step in between.  From Python the same takes about 5 us more per call (tensor attributes
// read one by one, torch.empty, a Stream object, ctypes), more than the kernel of a small projection: 1024 x 4096 with one
// request, called over and over, 9.1 -> 4.4 us a call (its kernel 2.8), the four calls of a Llama-3-8B block's linear layers with four
// requests 53 -> 30 us.
//
// Every function takes the call only if everything about it is as it should be (plain tensors, ints, lists, dicts; several matrices only with
// new results), and returns None otherwise: the Python code behind it then makes the same checks again and makes the call, or raises what it always raised.  Nothing is kept between calls.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <ATen/PythonTorchFunctionTLS.h>
#include <ATen/ops/empty.h>
#include <c10/hip/HIPStream.h>
#include <torch/csrc/Dtype.h>
#include <torch/csrc/autograd/python_variable.h>

#include "bcq.h"

namespace {

decltype(&bcq_gemv_offset) g_gemv = nullptr;
decltype(&bcq_gemv_multi) g_multi = nullptr;
decltype(&bcq_gemm_mixed) g_mixed = nullptr;
decltype(&bcq_gemm_mixed_offset) g_mixed_offset = nullptr;
decltype(&bcq_int8_quantize) g_int8_quantize = nullptr;
decltype(&bcq_int8_gemm) g_int8_gemm = nullptr;
decltype(&bcq_int8_gated) g_int8_gated = nullptr;
decltype(&bcq_int8_backward_workspace) g_int8_workspace = nullptr;
decltype(&bcq_int8_gemm_backward) g_int8_gemm_backward = nullptr;
decltype(&bcq_int8_gated_backward) g_int8_gated_backward = nullptr;
PyObject *g_error = nullptr;            // the exception class: (status, where)

// A plain tensor on the GPU, contiguous, of this type; nullptr otherwise.  (Subclasses, wrappers and tensors without storage go the Python way.)
const at::Tensor *gpu_tensor(PyObject *o, at::ScalarType type)
{
    if (!THPVariable_CheckExact(o)) return nullptr;
    const at::Tensor &t = THPVariable_Unpack(o);
    if (!t.defined() || !t.is_cuda() || t.scalar_type() != type || t.layout() != at::kStrided || !t.has_storage() || !t.is_contiguous()) return nullptr;
    return &t;
}

bool whole(PyObject *o, long &v)
{
    if (!PyLong_CheckExact(o)) return false;
    v = PyLong_AsLong(o);
    if (v == -1 && PyErr_Occurred()) {
        PyErr_Clear();
        return false;
    }
    return v >= 0 && v <= (1L << 30);
}

void *stream() { return c10::hip::getCurrentHIPStream().stream(); }

// other Python threads run while memory is allocated and kernels are launched, as they do during torch.empty and a ctypes call
struct WithoutGil {
    PyThreadState *state = PyEval_SaveThread();
    ~WithoutGil() { PyEval_RestoreThread(state); }
};

at::Tensor output(const at::Tensor &x, at::IntArrayRef sizes, at::ScalarType type)
{
    WithoutGil released;
    return at::empty(sizes, at::TensorOptions().dtype(type).device(x.device()));
}

template <typename F, typename... Args>
int launch(F f, Args... args)
{
    WithoutGil released;
    return f(args...);
}

// the result object, or the library's error
PyObject *finish(int status, const char *where, PyObject *y)
{
    if (status == 0) return y;
    Py_DECREF(y);
    if (PyObject *e = PyObject_CallFunction(g_error, "is", status, where)) {
        PyErr_SetObject(g_error, e);
        Py_DECREF(e);
    }
    return nullptr;
}

// planes [>= p][m][n/32], int32
const at::Tensor *planes_of(PyObject *o, int64_t &m, int64_t &n)
{
    const at::Tensor *t = gpu_tensor(o, at::kInt);
    if (!t || t->dim() != 3) return nullptr;
    m = t->size(1);
    n = t->size(2) * 32;
    return t;
}

bool scales_fit(const at::Tensor *t, int64_t p, int64_t m, int64_t ngroups)
{
    return t && t->dim() == 3 && t->size(0) == p && t->size(1) == m && t->size(2) == ngroups;
}

bool matrix_fits(const at::Tensor *t, int64_t rows, int64_t cols) { return t && t->dim() == 2 && t->size(0) == rows && t->size(1) == cols; }

const bcq_half *half(const at::Tensor *t) { return static_cast<const bcq_half *>(t->const_data_ptr()); }

// y: the caller's tensor, or a new one; nullptr where the caller's does not fit
PyObject *result(PyObject *given, const at::Tensor &x, int64_t batch, int64_t m, bcq_half *&ptr)
{
    if (given == Py_None) {
        at::Tensor y = output(x, {batch, m}, at::kHalf);
        ptr = static_cast<bcq_half *>(y.mutable_data_ptr());
        return THPVariable_Wrap(std::move(y));
    }
    const at::Tensor *y = gpu_tensor(given, at::kHalf);
    if (!matrix_fits(y, batch, m)) return nullptr;
    ptr = static_cast<bcq_half *>(y->mutable_data_ptr());
    Py_INCREF(given);
    return given;
}

// what the Python code would not get either: fall back to it and let it say so
template <typename F>
PyObject *guarded(F f)
{
    try {
        if (at::impl::torch_function_mode_enabled()) Py_RETURN_NONE;
        return f();
    } catch (...) {
        PyErr_Clear();
        Py_RETURN_NONE;
    }
}

// gemv(planes, scales_p, p, x, y, group, offsets)
PyObject *gemv(PyObject *, PyObject *const *a, Py_ssize_t count)
{
    if (count != 7 || !g_gemv) Py_RETURN_NONE;
    return guarded([&]() -> PyObject * {
        long p, group;
        int64_t m, n;
        const at::Tensor *planes = planes_of(a[0], m, n), *scales = gpu_tensor(a[1], at::kHalf), *x = gpu_tensor(a[3], at::kHalf);
        if (!planes || !x || x->dim() != 2 || !whole(a[2], p) || !whole(a[5], group) || group == 0) Py_RETURN_NONE;
        const int64_t batch = x->size(0);
        if (x->size(1) != n || batch > (1 << 30) || !scales_fit(scales, p, m, n / group) || planes->size(0) < p) Py_RETURN_NONE;
        const at::Tensor *offsets = nullptr;
        if (a[6] != Py_None) {
            offsets = gpu_tensor(a[6], at::kHalf);
            if (!matrix_fits(offsets, m, n / group)) Py_RETURN_NONE;
        }
        bcq_half *to = nullptr;
        PyObject *y = result(a[4], *x, batch, m, to);
        if (!y) Py_RETURN_NONE;
        const int status = launch(g_gemv, static_cast<const uint32_t *>(planes->const_data_ptr()), half(scales), offsets ? half(offsets) : nullptr, (int)p,
                                  half(x), to, m, n, (int)batch, (int)group, stream());
        return finish(status, offsets ? "bcq_gemv_offset" : "bcq_gemv", y);
    });
}

// gemv_multi(planes, scales_p, p, x, group): lists of the matrices, new outputs
PyObject *gemv_multi(PyObject *, PyObject *const *a, Py_ssize_t count)
{
    if (count != 5 || !g_multi) Py_RETURN_NONE;
    return guarded([&]() -> PyObject * {
        long p, group;
        const at::Tensor *x = gpu_tensor(a[3], at::kHalf);
        if (!PyList_CheckExact(a[0]) || !PyList_CheckExact(a[1]) || !x || x->dim() != 2 || !whole(a[2], p) || !whole(a[4], group) || group == 0)
            Py_RETURN_NONE;
        const Py_ssize_t k = PyList_GET_SIZE(a[0]);
        if (k < 1 || k > BCQ_MAX_MULTI || PyList_GET_SIZE(a[1]) != k) Py_RETURN_NONE;
        const int64_t batch = x->size(0), n = x->size(1);
        if (batch > (1 << 30)) Py_RETURN_NONE;
        const uint32_t *planes[BCQ_MAX_MULTI];
        const bcq_half *scales[BCQ_MAX_MULTI];
        int64_t ms[BCQ_MAX_MULTI];
        for (Py_ssize_t i = 0; i < k; ++i) {
            int64_t wide;
            const at::Tensor *w = planes_of(PyList_GET_ITEM(a[0], i), ms[i], wide), *s = gpu_tensor(PyList_GET_ITEM(a[1], i), at::kHalf);
            if (!w || wide != n || w->size(0) < p || !scales_fit(s, p, ms[i], n / group)) Py_RETURN_NONE;
            planes[i] = static_cast<const uint32_t *>(w->const_data_ptr());
            scales[i] = half(s);
        }
        PyObject *ys = PyList_New(k);
        if (!ys) return nullptr;
        bcq_half *to[BCQ_MAX_MULTI];
        for (Py_ssize_t i = 0; i < k; ++i) {
            PyObject *y = nullptr;
            try {
                y = result(Py_None, *x, batch, ms[i], to[i]);
            } catch (...) {
            }
            if (!y) {
                PyErr_Clear();
                Py_DECREF(ys);
                Py_RETURN_NONE;
            }
            PyList_SET_ITEM(ys, i, y);
        }
        return finish(launch(g_multi, (int)k, planes, scales, ms, to, (int)p, half(x), n, (int)batch, (int)group, stream()), "bcq_gemv_multi", ys);
    });
}

// sets by precision: a dict of whole numbers to tensors, their pointers in by_p[1 .. p_max]
template <typename Fits>
bool sets_of(PyObject *dict, int64_t p_max, const bcq_half **by_p, Fits fits)
{
    PyObject *key, *value;
    Py_ssize_t pos = 0;
    while (PyDict_Next(dict, &pos, &key, &value)) {
        long q;
        if (!whole(key, q) || q < 1 || q > p_max) return false;
        const at::Tensor *t = gpu_tensor(value, at::kHalf);
        if (!fits(t, q)) return false;
        by_p[q] = half(t);
    }
    return true;
}

// gemm_mixed(planes, scales_by_p, p_req, x, y, group, offsets_by_p)
PyObject *gemm_mixed(PyObject *, PyObject *const *a, Py_ssize_t count)
{
    if (count != 7 || !g_mixed) Py_RETURN_NONE;
    return guarded([&]() -> PyObject * {
        long group;
        int64_t m, n;
        const at::Tensor *planes = planes_of(a[0], m, n), *p_req = gpu_tensor(a[2], at::kInt), *x = gpu_tensor(a[3], at::kHalf);
        if (!planes || !p_req || !x || x->dim() != 2 || !PyDict_CheckExact(a[1]) || !whole(a[5], group) || group == 0) Py_RETURN_NONE;
        const int64_t p_max = planes->size(0), batch = x->size(0);
        if (p_max < 1 || p_max > BCQ_MAX_PLANES || batch > (1 << 30) || x->size(1) != n || p_req->dim() != 1 || p_req->size(0) != batch) Py_RETURN_NONE;
        const bcq_half *scales[BCQ_MAX_PLANES + 1] = {}, *offsets[BCQ_MAX_PLANES + 1] = {};
        const int64_t ngroups = n / group;
        if (!sets_of(a[1], p_max, scales, [&](const at::Tensor *t, long q) { return scales_fit(t, q, m, ngroups); })) Py_RETURN_NONE;
        bool with_offsets = false;
        if (a[6] != Py_None) {
            if (!PyDict_CheckExact(a[6])) Py_RETURN_NONE;
            with_offsets = PyDict_Size(a[6]) > 0;
            if (!sets_of(a[6], p_max, offsets, [&](const at::Tensor *t, long) { return matrix_fits(t, m, ngroups); })) Py_RETURN_NONE;
        }
        bcq_half *to = nullptr;
        PyObject *y = result(a[4], *x, batch, m, to);
        if (!y) Py_RETURN_NONE;
        const uint32_t *w = static_cast<const uint32_t *>(planes->const_data_ptr());
        const int32_t *req = static_cast<const int32_t *>(p_req->const_data_ptr());
        if (with_offsets)
            return finish(launch(g_mixed_offset, w, scales, offsets, req, (int)p_max, half(x), to, m, n, (int)batch, (int)group, stream()),
                          "bcq_gemm_mixed_offset", y);
        return finish(launch(g_mixed, w, scales, req, (int)p_max, half(x), to, m, n, (int)batch, (int)group, stream()), "bcq_gemm_mixed", y);
    });
}

// A 16-bit type by its torch name; false otherwise.
bool type_of(at::ScalarType scalar, int &type)
{
    if (scalar != at::kHalf && scalar != at::kBFloat16) return false;
    type = scalar == at::kHalf ? BCQ_FLOAT16 : BCQ_BFLOAT16;
    return true;
}

// Tensors of the 8-bit operators live on one device, the current one.
struct OneDevice {
    c10::Device device;
    bool same = true;
    explicit OneDevice(const at::Tensor &first) : device(first.device()) { same = device.index() == c10::hip::current_device(); }
    const at::Tensor *take(PyObject *o, at::ScalarType type)
    {
        const at::Tensor *t = gpu_tensor(o, type);
        if (t && t->device() != device) t = nullptr;
        if (!t) same = false;
        return t;
    }
    // [rows] or [rows][cols], the caller's or a new one; nullptr where the caller's does not fit
    PyObject *result(PyObject *given, const at::Tensor &like, at::ScalarType type, at::IntArrayRef sizes, void *&ptr)
    {
        if (given == Py_None) {
            at::Tensor y = output(like, sizes, type);
            ptr = y.mutable_data_ptr();
            return THPVariable_Wrap(std::move(y));
        }
        const at::Tensor *y = take(given, type);
        if (!y || y->sizes() != sizes) return nullptr;
        ptr = y->mutable_data_ptr();
        Py_INCREF(given);
        return given;
    }
};

// int8_quantize(x, q, scales) -> (codes, scales)
PyObject *int8_quantize(PyObject *, PyObject *const *a, Py_ssize_t count)
{
    if (count != 3 || !g_int8_quantize) Py_RETURN_NONE;
    return guarded([&]() -> PyObject * {
        const at::Tensor *x = gpu_tensor(a[0], at::kHalf);
        if (!x) x = gpu_tensor(a[0], at::kBFloat16);
        int type;
        if (!x || x->dim() != 2 || !type_of(x->scalar_type(), type)) Py_RETURN_NONE;
        OneDevice on(*x);
        if (!on.same) Py_RETURN_NONE;
        const int64_t rows = x->size(0), n = x->size(1);
        void *q_to = nullptr, *s_to = nullptr;
        PyObject *q = on.result(a[1], *x, at::kChar, {rows, n}, q_to);
        if (!q) Py_RETURN_NONE;
        PyObject *s = nullptr;
        try {
            s = on.result(a[2], *x, at::kFloat, {rows}, s_to);
        } catch (...) {
        }
        PyObject *both = s ? PyTuple_New(2) : nullptr;
        if (!both) {
            PyErr_Clear();
            Py_DECREF(q);
            Py_XDECREF(s);
            Py_RETURN_NONE;
        }
        PyTuple_SET_ITEM(both, 0, q);
        PyTuple_SET_ITEM(both, 1, s);
        return finish(launch(g_int8_quantize, x->const_data_ptr(), type, static_cast<int8_t *>(q_to), static_cast<float *>(s_to), rows, n, stream()),
                      "bcq_int8_quantize", both);
    });
}

const int8_t *codes(const at::Tensor *t) { return static_cast<const int8_t *>(t->const_data_ptr()); }
const float *floats(const at::Tensor *t) { return static_cast<const float *>(t->const_data_ptr()); }

// The codes of some tokens and `mats` matrices, each with its scales: a[0], a[1], then pairs.  False where they do not fit together.
bool int8_operands(OneDevice &on, PyObject *const *a, int mats, const at::Tensor **t, int64_t &m, int64_t &n, int64_t &tokens)
{
    for (int k = 0; k < 2 + 2 * mats; ++k)
        if (!(t[k] = on.take(a[k], k & 1 ? at::kFloat : at::kChar))) return false;
    if (t[0]->dim() != 2 || t[2]->dim() != 2) return false;
    tokens = t[0]->size(0);
    n = t[0]->size(1);
    m = t[2]->size(0);
    if (t[1]->dim() != 1 || t[1]->size(0) != tokens) return false;
    for (int k = 2; k < 2 + 2 * mats; k += 2)
        if (!matrix_fits(t[k], m, n) || t[k + 1]->dim() != 1 || t[k + 1]->size(0) != m) return false;
    return on.same;
}

// int8_gemm(q, token_scales, w, channel_scales, dtype, y)
PyObject *int8_gemm(PyObject *, PyObject *const *a, Py_ssize_t count)
{
    if (count != 6 || !g_int8_gemm) Py_RETURN_NONE;
    return guarded([&]() -> PyObject * {
        int type;
        const at::Tensor *q = gpu_tensor(a[0], at::kChar), *t[4];
        if (!q || !THPDtype_Check(a[4]) || !type_of(reinterpret_cast<THPDtype *>(a[4])->scalar_type, type)) Py_RETURN_NONE;
        OneDevice on(*q);
        int64_t m, n, tokens;
        if (!int8_operands(on, a, 1, t, m, n, tokens)) Py_RETURN_NONE;
        void *to = nullptr;
        PyObject *y = on.result(a[5], *q, type == BCQ_FLOAT16 ? at::kHalf : at::kBFloat16, {tokens, m}, to);
        if (!y) Py_RETURN_NONE;
        return finish(launch(g_int8_gemm, codes(t[0]), floats(t[1]), codes(t[2]), floats(t[3]), to, type, m, n, tokens, stream()), "bcq_int8_gemm", y);
    });
}

// int8_gated(q, token_scales, w_gate, gate_scales, w_up, up_scales, activation, dtype, h)
PyObject *int8_gated(PyObject *, PyObject *const *a, Py_ssize_t count)
{
    if (count != 9 || !g_int8_gated) Py_RETURN_NONE;
    return guarded([&]() -> PyObject * {
        int type;
        const at::Tensor *q = gpu_tensor(a[0], at::kChar), *t[6];
        if (!q || !PyUnicode_CheckExact(a[6]) || !THPDtype_Check(a[7]) || !type_of(reinterpret_cast<THPDtype *>(a[7])->scalar_type, type)) Py_RETURN_NONE;
        const bool silu = PyUnicode_CompareWithASCIIString(a[6], "silu") == 0;
        if (!silu && PyUnicode_CompareWithASCIIString(a[6], "gelu") != 0) Py_RETURN_NONE;
        OneDevice on(*q);
        int64_t m, n, tokens;
        if (!int8_operands(on, a, 2, t, m, n, tokens)) Py_RETURN_NONE;
        void *to = nullptr;
        PyObject *h = on.result(a[8], *q, type == BCQ_FLOAT16 ? at::kHalf : at::kBFloat16, {tokens, m}, to);
        if (!h) Py_RETURN_NONE;
        return finish(launch(g_int8_gated, codes(t[0]), floats(t[1]), codes(t[2]), floats(t[3]), codes(t[4]), floats(t[5]),
                             (int)(silu ? BCQ_ACT_SILU : BCQ_ACT_GELU), to, type, m, n, tokens, stream()),
                      "bcq_int8_gated", h);
    });
}

// What the backward calls share: the gradient, new results (dx, then the gradients of the scales, a tuple) and the workspace; the call itself is `f`'s.
template <typename F>
PyObject *int8_backward(PyObject *const *a, int mats, const char *where, F f)
{
    int type;
    const at::Tensor *dy = gpu_tensor(a[0], at::kHalf), *t[6];
    if (!dy) dy = gpu_tensor(a[0], at::kBFloat16);
    if (!dy || !type_of(dy->scalar_type(), type)) Py_RETURN_NONE;
    OneDevice on(*dy);
    int64_t m, n, tokens;
    if (!int8_operands(on, a + 1, mats, t, m, n, tokens) || !matrix_fits(dy, tokens, m)) Py_RETURN_NONE;
    const int64_t size = g_int8_workspace(mats, m, n, tokens);
    if (size < 0) Py_RETURN_NONE;
    const at::Tensor workspace = output(*dy, {size}, at::kByte);
    at::Tensor dx = output(*dy, {tokens, n}, dy->scalar_type()), dscales[2];
    for (int k = 0; k < mats; ++k) dscales[k] = output(*dy, {m}, at::kFloat);
    const int status = f(dy->const_data_ptr(), t, dx.mutable_data_ptr(), static_cast<float *>(dscales[0].mutable_data_ptr()),
                         mats == 2 ? static_cast<float *>(dscales[1].mutable_data_ptr()) : nullptr, type, m, n, tokens, workspace.mutable_data_ptr(), size);
    PyObject *results = PyTuple_New(1 + mats);
    if (!results) return nullptr;
    for (int k = 0; k <= mats; ++k) {
        PyObject *r = THPVariable_Wrap(k == 0 ? std::move(dx) : std::move(dscales[k - 1]));
        if (!r) {
            Py_DECREF(results);
            return nullptr;
        }
        PyTuple_SET_ITEM(results, k, r);
    }
    return finish(status, where, results);
}

// int8_gemm_backward(dy, q, token_scales, w, channel_scales) -> (dx, dchannel_scales)
PyObject *int8_gemm_backward(PyObject *, PyObject *const *a, Py_ssize_t count)
{
    if (count != 5 || !g_int8_gemm_backward) Py_RETURN_NONE;
    return guarded([&]() -> PyObject * {
        return int8_backward(a, 1, "bcq_int8_gemm_backward",
                             [&](const void *dy, const at::Tensor **t, void *dx, float *d0, float *, int type, int64_t m, int64_t n, int64_t tokens,
                                 void *workspace, int64_t size) {
                                 return launch(g_int8_gemm_backward, dy, codes(t[0]), floats(t[1]), codes(t[2]), floats(t[3]), dx, d0, type, m, n, tokens,
                                               workspace, size, stream());
                             });
    });
}

// int8_gated_backward(dh, q, token_scales, w_gate, gate_scales, w_up, up_scales, activation) -> (dx, dgate_scales, dup_scales)
PyObject *int8_gated_backward(PyObject *, PyObject *const *a, Py_ssize_t count)
{
    if (count != 8 || !g_int8_gated_backward || !PyUnicode_CheckExact(a[7])) Py_RETURN_NONE;
    return guarded([&]() -> PyObject * {
        const bool silu = PyUnicode_CompareWithASCIIString(a[7], "silu") == 0;
        if (!silu && PyUnicode_CompareWithASCIIString(a[7], "gelu") != 0) Py_RETURN_NONE;
        return int8_backward(a, 2, "bcq_int8_gated_backward",
                             [&](const void *dh, const at::Tensor **t, void *dx, float *d0, float *d1, int type, int64_t m, int64_t n, int64_t tokens,
                                 void *workspace, int64_t size) {
                                 return launch(g_int8_gated_backward, dh, codes(t[0]), floats(t[1]), codes(t[2]), floats(t[3]), codes(t[4]), floats(t[5]),
                                               (int)(silu ? BCQ_ACT_SILU : BCQ_ACT_GELU), dx, d0, d1, type, m, n, tokens, workspace, size, stream());
                             });
    });
}

// bind_int8(quantize, gemm, gated, backward_workspace, gemm_backward, gated_backward): likewise the 8-bit operators
PyObject *bind_int8(PyObject *, PyObject *args)
{
    unsigned long long f[6];
    if (!PyArg_ParseTuple(args, "KKKKKK", &f[0], &f[1], &f[2], &f[3], &f[4], &f[5])) return nullptr;
    g_int8_quantize = reinterpret_cast<decltype(g_int8_quantize)>(f[0]);
    g_int8_gemm = reinterpret_cast<decltype(g_int8_gemm)>(f[1]);
    g_int8_gated = reinterpret_cast<decltype(g_int8_gated)>(f[2]);
    g_int8_workspace = reinterpret_cast<decltype(g_int8_workspace)>(f[3]);
    g_int8_gemm_backward = reinterpret_cast<decltype(g_int8_gemm_backward)>(f[4]);
    g_int8_gated_backward = reinterpret_cast<decltype(g_int8_gated_backward)>(f[5]);
    Py_RETURN_NONE;
}

// bind(gemv_offset, gemv_multi, gemm_mixed, gemm_mixed_offset, error): addresses of the C ABI's functions in the library that is loaded
PyObject *bind(PyObject *, PyObject *args)
{
    unsigned long long f[4];
    PyObject *error;
    if (!PyArg_ParseTuple(args, "KKKKO", &f[0], &f[1], &f[2], &f[3], &error)) return nullptr;
    g_gemv = reinterpret_cast<decltype(g_gemv)>(f[0]);
    g_multi = reinterpret_cast<decltype(g_multi)>(f[1]);
    g_mixed = reinterpret_cast<decltype(g_mixed)>(f[2]);
    g_mixed_offset = reinterpret_cast<decltype(g_mixed_offset)>(f[3]);
    Py_INCREF(error);
    Py_XSETREF(g_error, error);
    Py_RETURN_NONE;
}

PyMethodDef g_methods[] = {{"gemv", (PyCFunction)(void (*)(void))gemv, METH_FASTCALL, nullptr},
                           {"gemv_multi", (PyCFunction)(void (*)(void))gemv_multi, METH_FASTCALL, nullptr},
                           {"gemm_mixed", (PyCFunction)(void (*)(void))gemm_mixed, METH_FASTCALL, nullptr},
                           {"int8_quantize", (PyCFunction)(void (*)(void))int8_quantize, METH_FASTCALL, nullptr},
                           {"int8_gemm", (PyCFunction)(void (*)(void))int8_gemm, METH_FASTCALL, nullptr},
                           {"int8_gated", (PyCFunction)(void (*)(void))int8_gated, METH_FASTCALL, nullptr},
                           {"int8_gemm_backward", (PyCFunction)(void (*)(void))int8_gemm_backward, METH_FASTCALL, nullptr},
                           {"int8_gated_backward", (PyCFunction)(void (*)(void))int8_gated_backward, METH_FASTCALL, nullptr},
                           {"bind", bind, METH_VARARGS, nullptr},
                           {"bind_int8", bind_int8, METH_VARARGS, nullptr},
                           {nullptr, nullptr, 0, nullptr}};
PyModuleDef g_module = {PyModuleDef_HEAD_INIT, "_bcq_host", nullptr, -1, g_methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

// the torch this was built against, as torch.__version__ has it: another one's tensors may be laid out differently
constexpr char kBuiltFor[] = "built for torch " BCQ_TORCH_VERSION;

PyMODINIT_FUNC PyInit__bcq_host(void)
{
    PyObject *module = PyModule_Create(&g_module);
    if (module && PyModule_AddStringConstant(module, "torch_version", kBuiltFor + sizeof "built for torch " - 1) != 0) Py_CLEAR(module);
    return module;
}
