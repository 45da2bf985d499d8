// CPython extension: the hot entry points called with ordinary arguments (dense device tensors of the expected types, tuples or
// lists of plain integers, the current stream) without ctypes and without a Python object per argument.
//
// Every function returns the library's status, or None where an argument is anything else; the caller then takes the general
// path, which accepts what it always accepted and raises what it always raised.  Nothing is launched before every argument has
// been looked at.
//
// What bounds a small layer is the host: five launches of 2.4 us each and, through ctypes, as much again in Python.  us per call,
// host alone, ctypes against this: sta_tile_permute 5.3, 3.05; sta_forward of 2 heads 7.5, 3.5, of 24 11.4, 3.9.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <ATen/core/Tensor.h>
#include <torch/csrc/autograd/python_variable.h>

#include <cstdint>

#include "../../include/sta.h"

namespace {

using PermuteFn = int (*)(const void *, void *, int, int, int, int, int, const int *, const int *, void *);
using ForwardFn = int (*)(const void *, const void *, const void *, void *, int, int, int, const int *, const int *, const int *,
                          float, void *, size_t, void *);
using ForwardLseFn = int (*)(const void *, const void *, const void *, void *, float *, int, int, int, const int *, const int *,
                             const int *, float, void *);
using BackwardFn = int (*)(const void *, const void *, const void *, const void *, const void *, const float *, void *, void *,
                           void *, int, int, int, const int *, const int *, const int *, float, void *, size_t, void *);

struct Entries {
    PermuteFn tile_permute, untile;
    ForwardFn forward;
    ForwardLseFn forward_lse;
    BackwardFn backward;
} entries = {};
PyObject *current_device, *current_raw_stream;      // torch's own, called for every launch

constexpr int kMaxHeads = 1024;                     // more go the general way
enum { kBf16 = 0, kF32 = 1 };                       // STA_BF16, STA_F32

// A dense device tensor as the kernels take it.
struct View {
    const at::Tensor *t;
    void *ptr;
};
bool dense(PyObject *o, View &v)
{
    if (!THPVariable_CheckExact(o)) return false;
    v.t = &THPVariable_Unpack(o);
    if (!v.t->is_cuda() || !v.t->is_contiguous() || v.t->layout() != at::kStrided) return false;
    v.ptr = v.t->data_ptr();                        // throws for tensors without storage
    return true;
}
bool same_shape4(const View *v, int n)
{
    const auto shape = v[0].t->sizes();
    if (shape.size() != 4) return false;
    for (int i = 0; i < 4; ++i)
        if (shape[i] > INT32_MAX) return false;
    for (int i = 1; i < n; ++i)
        if (v[i].t->sizes() != shape) return false;
    return true;
}
bool all_bf16(const View *v, int n)
{
    for (int i = 0; i < n; ++i)
        if (v[i].t->scalar_type() != at::kBFloat16) return false;
    return true;
}
bool dtype_code(const View &v, int &code)
{
    const auto type = v.t->scalar_type();
    code = type == at::kBFloat16 ? kBf16 : kF32;
    return type == at::kBFloat16 || type == at::kFloat;
}

// n plain integers from a tuple or a list.
bool ints(PyObject *o, Py_ssize_t n, int *out)
{
    PyObject **items;
    if (PyTuple_CheckExact(o)) {
        if (PyTuple_GET_SIZE(o) != n) return false;
        items = &PyTuple_GET_ITEM(o, 0);
    } else if (PyList_CheckExact(o)) {
        if (PyList_GET_SIZE(o) != n) return false;
        items = &PyList_GET_ITEM(o, 0);
    } else {
        return false;
    }
    for (Py_ssize_t i = 0; i < n; ++i) {
        if (!PyLong_CheckExact(items[i])) return false;
        int overflow;
        const long x = PyLong_AsLongAndOverflow(items[i], &overflow);
        if (overflow != 0 || x < INT32_MIN || x > INT32_MAX) return false;
        out[i] = (int)x;
    }
    return true;
}
bool windows(PyObject *o, int64_t heads, int *out)
{
    if (heads > kMaxHeads) return false;
    PyObject **items;
    if (PyList_CheckExact(o) && PyList_GET_SIZE(o) == heads) items = &PyList_GET_ITEM(o, 0);
    else if (PyTuple_CheckExact(o) && PyTuple_GET_SIZE(o) == heads) items = &PyTuple_GET_ITEM(o, 0);
    else return false;
    for (int64_t h = 0; h < heads; ++h)
        if (!ints(items[h], 3, out + 3 * h)) return false;
    return true;
}
bool number(PyObject *o, float &out)
{
    if (!PyFloat_CheckExact(o)) return false;
    out = (float)PyFloat_AS_DOUBLE(o);
    return true;
}
bool tokens_match(int64_t n, const int *grid) { return n == (int64_t)grid[0] * grid[1] * grid[2]; }

// The current stream of the current device; false with an exception set.
bool stream_of(void *&stream)
{
    PyObject *device = PyObject_CallNoArgs(current_device);
    if (!device) return false;
    PyObject *raw = PyObject_CallOneArg(current_raw_stream, device);
    Py_DECREF(device);
    if (!raw) return false;
    stream = PyLong_AsVoidPtr(raw);
    Py_DECREF(raw);
    return !PyErr_Occurred();
}

template <typename F>
PyObject *guarded(F &&f)
{
    try {
        return f();
    } catch (...) {                                 // a tensor that has no memory to point to: the general path says so
        PyErr_Clear();
        Py_RETURN_NONE;
    }
}
template <typename F>
PyObject *status_of(F &&launch)
{
    int status;
    Py_BEGIN_ALLOW_THREADS
    status = launch();
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(status);
}

// (src, dst, grid, tile)
PyObject *permute(PermuteFn fn, PyObject *const *args, Py_ssize_t n)
{
    return guarded([&]() -> PyObject * {
        View v[2];
        int grid[3], tile[3], src_type, dst_type;
        void *stream;
        if (!fn || n != 4 || !dense(args[0], v[0]) || !dense(args[1], v[1]) || !same_shape4(v, 2) || !dtype_code(v[0], src_type) ||
            !dtype_code(v[1], dst_type) || !ints(args[2], 3, grid) || !ints(args[3], 3, tile) || !tokens_match(v[0].t->size(2), grid))
            Py_RETURN_NONE;
        if (!stream_of(stream)) return nullptr;
        const int B = (int)v[0].t->size(0), H = (int)v[0].t->size(1), D = (int)v[0].t->size(3);
        return status_of([&]() { return fn(v[0].ptr, v[1].ptr, src_type, dst_type, B, H, D, grid, tile, stream); });
    });
}
PyObject *py_tile_permute(PyObject *, PyObject *const *args, Py_ssize_t n) { return permute(entries.tile_permute, args, n); }
PyObject *py_untile(PyObject *, PyObject *const *args, Py_ssize_t n) { return permute(entries.untile, args, n); }

// (q, k, v, o, grid, tile, windows, scale, workspace or None)
PyObject *py_forward(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    return guarded([&]() -> PyObject * {
        View v[4], ws = {nullptr, nullptr};
        int grid[3], tile[3], win[3 * kMaxHeads];
        float scale;
        void *stream;
        if (!entries.forward || n != 9) Py_RETURN_NONE;
        for (int i = 0; i < 4; ++i)
            if (!dense(args[i], v[i])) Py_RETURN_NONE;
        if (!same_shape4(v, 4) || !all_bf16(v, 4) || !ints(args[4], 3, grid) || !ints(args[5], 3, tile) ||
            !tokens_match(v[0].t->size(2), grid) || !windows(args[6], v[0].t->size(1), win) || !number(args[7], scale) ||
            (args[8] != Py_None && !dense(args[8], ws)))
            Py_RETURN_NONE;
        const size_t ws_bytes = ws.t ? ws.t->numel() * ws.t->element_size() : 0;
        if (!stream_of(stream)) return nullptr;
        const int B = (int)v[0].t->size(0), H = (int)v[0].t->size(1), D = (int)v[0].t->size(3);
        return status_of([&]() {
            return entries.forward(v[0].ptr, v[1].ptr, v[2].ptr, v[3].ptr, B, H, D, grid, tile, win, scale, ws.ptr, ws_bytes, stream);
        });
    });
}

// lse: float32 [B, H, N] that goes with tensors of shape [B, H, N, D]
bool lse_of(PyObject *o, const View &like, View &lse)
{
    return dense(o, lse) && lse.t->scalar_type() == at::kFloat && lse.t->dim() == 3 && lse.t->sizes() == like.t->sizes().slice(0, 3);
}

// (q, k, v, o, lse, grid, tile, windows, scale)
PyObject *py_forward_lse(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    return guarded([&]() -> PyObject * {
        View v[4], lse;
        int grid[3], tile[3], win[3 * kMaxHeads];
        float scale;
        void *stream;
        if (!entries.forward_lse || n != 9) Py_RETURN_NONE;
        for (int i = 0; i < 4; ++i)
            if (!dense(args[i], v[i])) Py_RETURN_NONE;
        if (!same_shape4(v, 4) || !all_bf16(v, 4) || !lse_of(args[4], v[0], lse) || !ints(args[5], 3, grid) || !ints(args[6], 3, tile) ||
            !tokens_match(v[0].t->size(2), grid) || !windows(args[7], v[0].t->size(1), win) || !number(args[8], scale))
            Py_RETURN_NONE;
        if (!stream_of(stream)) return nullptr;
        const int B = (int)v[0].t->size(0), H = (int)v[0].t->size(1), D = (int)v[0].t->size(3);
        return status_of([&]() {
            return entries.forward_lse(v[0].ptr, v[1].ptr, v[2].ptr, v[3].ptr, static_cast<float *>(lse.ptr), B, H, D, grid, tile, win,
                                       scale, stream);
        });
    });
}

// (q, k, v, o, d_o, lse, d_q, d_k, d_v, grid, tile, windows, workspace, scale)
PyObject *py_backward(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    return guarded([&]() -> PyObject * {
        View v[8], lse, ws;
        int grid[3], tile[3], win[3 * kMaxHeads];
        float scale;
        void *stream;
        if (!entries.backward || n != 14) Py_RETURN_NONE;
        for (int i = 0; i < 8; ++i)
            if (!dense(args[i < 5 ? i : i + 1], v[i])) Py_RETURN_NONE;
        if (!same_shape4(v, 8) || !all_bf16(v, 8) || !lse_of(args[5], v[0], lse) || !ints(args[9], 3, grid) || !ints(args[10], 3, tile) ||
            !tokens_match(v[0].t->size(2), grid) || !windows(args[11], v[0].t->size(1), win) || !dense(args[12], ws) ||
            !number(args[13], scale))
            Py_RETURN_NONE;
        const size_t ws_bytes = ws.t->numel() * ws.t->element_size();
        if (!stream_of(stream)) return nullptr;
        const int B = (int)v[0].t->size(0), H = (int)v[0].t->size(1), D = (int)v[0].t->size(3);
        return status_of([&]() {
            return entries.backward(v[0].ptr, v[1].ptr, v[2].ptr, v[3].ptr, v[4].ptr, static_cast<const float *>(lse.ptr), v[5].ptr,
                                    v[6].ptr, v[7].ptr, B, H, D, grid, tile, win, scale, ws.ptr, ws_bytes, stream);
        });
    });
}

// ---- rows of heads and packed sequences: strided device tensors, one launch each; us per call, host alone, ctypes against this:
// sta_qk_norm_rope of q, k and v 10.7, 4.7; sta_packed_forward 8.8, 3.9; sta_rope of two tensors 8.7, 3.8
struct LayerEntries {
    decltype(&sta_rope) rope;
    decltype(&sta_qk_norm_rope) norm_rope;
    decltype(&sta_qk_norm_rope_backward) norm_rope_backward;
    decltype(&sta_packed_forward) packed_forward;
    decltype(&sta_packed_backward) packed_backward;
} layers = {};

bool small(int64_t x) { return x <= INT32_MAX; }

// A device tensor [B, N, H, D] whose channels are adjacent.
bool head_rows(PyObject *o, int64_t B, int64_t N, int64_t D, sta_head_rows &r)
{
    if (!THPVariable_CheckExact(o)) return false;
    const at::Tensor &t = THPVariable_Unpack(o);
    if (!t.is_cuda() || t.layout() != at::kStrided || t.dim() != 4 || t.numel() == 0) return false;
    const auto size = t.sizes(), stride = t.strides();
    const auto type = t.scalar_type();
    if (size[0] != B || size[1] != N || size[3] != D || stride[3] != 1 || !small(size[2]) || (type != at::kBFloat16 && type != at::kFloat)) return false;
    r = {t.data_ptr(), stride[0], stride[1], stride[2], (int)size[2], type == at::kBFloat16 ? kBf16 : kF32};
    return true;
}
// B, N and D of the first tensor.
bool first_shape(PyObject *o, int64_t (&s)[3])
{
    if (!THPVariable_CheckExact(o)) return false;
    const at::Tensor &t = THPVariable_Unpack(o);
    if (t.dim() != 4) return false;
    s[0] = t.size(0); s[1] = t.size(1); s[2] = t.size(3);
    return small(s[0]) && small(s[1]) && small(s[2]);
}
// None, or (address of a sta_rotary, tokens its positions are for or -1, batch entries or -1)
bool rotary_of(PyObject *o, int64_t B, int64_t N, const sta_rotary *&out)
{
    out = nullptr;
    if (o == Py_None) return true;
    if (!PyTuple_CheckExact(o) || PyTuple_GET_SIZE(o) != 3) return false;
    const long long n = PyLong_AsLongLong(PyTuple_GET_ITEM(o, 1)), b = PyLong_AsLongLong(PyTuple_GET_ITEM(o, 2));
    out = static_cast<const sta_rotary *>(PyLong_AsVoidPtr(PyTuple_GET_ITEM(o, 0)));
    if (PyErr_Occurred()) {
        PyErr_Clear();
        return false;
    }
    return out != nullptr && (n < 0 || n == N) && (b < 0 || b == B);
}
// One dimension of n elements, dense; None: null.
bool vector(PyObject *o, int64_t n, at::ScalarType type, const void *&out)
{
    out = nullptr;
    if (o == Py_None) return true;
    View v;
    if (!dense(o, v) || v.t->dim() != 1 || v.t->size(0) != n || v.t->scalar_type() != type) return false;
    out = v.ptr;
    return out != nullptr || n == 0;
}
// The two weights, of one type.
bool weights(PyObject *a, PyObject *b, int64_t D, const void *(&w)[2], int &type)
{
    if (vector(a, D, at::kFloat, w[0]) && vector(b, D, at::kFloat, w[1])) {
        type = kF32;
        return true;
    }
    type = kBf16;
    return vector(a, D, at::kBFloat16, w[0]) && vector(b, D, at::kBFloat16, w[1]);
}
bool grid_tile(PyObject *g, PyObject *t, int (&grid)[3], int (&tile)[3])
{
    return (g == Py_None || ints(g, 3, grid)) && (t == Py_None || (g != Py_None && ints(t, 3, tile)));
}
bool scratch(PyObject *o, void *&ptr, size_t &bytes)
{
    ptr = nullptr;
    bytes = 0;
    if (o == Py_None) return true;
    View v;
    if (!dense(o, v)) return false;
    ptr = v.ptr;
    bytes = v.t->numel() * v.t->element_size();
    return true;
}
bool integer(PyObject *o, int &out)
{
    int overflow;
    if (!PyLong_CheckExact(o)) return false;
    const long x = PyLong_AsLongAndOverflow(o, &overflow);
    out = (int)x;
    return overflow == 0 && x >= INT32_MIN && x <= INT32_MAX;
}

// (inputs, outputs, rotary, inverse)
PyObject *py_rope(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    return guarded([&]() -> PyObject * {
        sta_head_rows in[3], out[3];
        PyObject **items[2];
        Py_ssize_t count[2];
        if (!layers.rope || n != 4 || !PyBool_Check(args[3])) Py_RETURN_NONE;
        for (int i = 0; i < 2; ++i) {
            if (PyTuple_CheckExact(args[i])) { items[i] = &PyTuple_GET_ITEM(args[i], 0); count[i] = PyTuple_GET_SIZE(args[i]); }
            else if (PyList_CheckExact(args[i])) { items[i] = &PyList_GET_ITEM(args[i], 0); count[i] = PyList_GET_SIZE(args[i]); }
            else Py_RETURN_NONE;
        }
        int64_t s[3];
        const sta_rotary *rotary;
        if (count[0] < 1 || count[0] > 3 || count[1] != count[0] || !first_shape(items[0][0], s) || !rotary_of(args[2], s[0], s[1], rotary) || !rotary)
            Py_RETURN_NONE;
        for (Py_ssize_t i = 0; i < count[0]; ++i)
            if (!head_rows(items[0][i], s[0], s[1], s[2], in[i]) || !head_rows(items[1][i], s[0], s[1], s[2], out[i])) Py_RETURN_NONE;
        const int inverse = args[3] == Py_True;
        void *stream;
        if (!stream_of(stream)) return nullptr;
        return status_of([&]() { return layers.rope(in, out, (int)count[0], (int)s[0], (int)s[1], (int)s[2], rotary, inverse, stream); });
    });
}

// (q, k, v, q_out, k_out, v_out, q_weight, k_weight, rotary, eps, grid, tile)
PyObject *py_norm_rope(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    return guarded([&]() -> PyObject * {
        sta_head_rows r[6];
        int64_t s[3];
        const sta_rotary *rotary;
        const void *w[2];
        int type, grid[3], tile[3];
        float eps;
        if (!layers.norm_rope || n != 12 || !first_shape(args[0], s) || !rotary_of(args[8], s[0], s[1], rotary) || !weights(args[6], args[7], s[2], w, type) ||
            !number(args[9], eps) || !grid_tile(args[10], args[11], grid, tile) || (args[2] == Py_None) != (args[5] == Py_None))
            Py_RETURN_NONE;
        for (int i = 0; i < 6; ++i)
            if (args[i] == Py_None ? i % 3 != 2 : !head_rows(args[i], s[0], s[1], s[2], r[i])) Py_RETURN_NONE;
        const bool values = args[2] != Py_None;
        void *stream;
        if (!stream_of(stream)) return nullptr;
        return status_of([&]() {
            return layers.norm_rope(&r[0], &r[1], values ? &r[2] : nullptr, &r[3], &r[4], values ? &r[5] : nullptr, w[0], w[1], type, eps, rotary, (int)s[0],
                                    (int)s[1], (int)s[2], args[10] == Py_None ? nullptr : grid, args[11] == Py_None ? nullptr : tile, stream);
        });
    });
}

// (q, k, d_q_out, d_k_out, d_v_out, d_q, d_k, d_v, q_weight, k_weight, d_q_weight, d_k_weight, rotary, workspace, eps, grid, tile)
PyObject *py_norm_rope_backward(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    return guarded([&]() -> PyObject * {
        sta_head_rows r[8];
        int64_t s[3];
        const sta_rotary *rotary;
        const void *w[2], *dw[2];
        int type, grid[3], tile[3];
        float eps;
        void *ws, *stream;
        size_t bytes;
        if (!layers.norm_rope_backward || n != 17 || !first_shape(args[0], s) || !rotary_of(args[12], s[0], s[1], rotary) ||
            !weights(args[8], args[9], s[2], w, type) || !vector(args[10], s[2], at::kFloat, dw[0]) || !vector(args[11], s[2], at::kFloat, dw[1]) ||
            !scratch(args[13], ws, bytes) || !number(args[14], eps) || !grid_tile(args[15], args[16], grid, tile) ||
            (args[4] == Py_None) != (args[7] == Py_None))
            Py_RETURN_NONE;
        for (int i = 0; i < 8; ++i)
            if (args[i] == Py_None ? i != 4 && i != 7 : !head_rows(args[i], s[0], s[1], s[2], r[i])) Py_RETURN_NONE;
        const bool values = args[4] != Py_None;
        if (!stream_of(stream)) return nullptr;
        return status_of([&]() {
            return layers.norm_rope_backward(&r[0], &r[1], &r[2], &r[3], values ? &r[4] : nullptr, &r[5], &r[6], values ? &r[7] : nullptr, w[0], w[1], type,
                                             static_cast<float *>(const_cast<void *>(dw[0])), static_cast<float *>(const_cast<void *>(dw[1])), eps, rotary,
                                             (int)s[0], (int)s[1], (int)s[2], args[15] == Py_None ? nullptr : grid, args[16] == Py_None ? nullptr : tile, ws,
                                             bytes, stream);
        });
    });
}

// A device tensor [tokens, H, D] of bf16 whose channels are adjacent.
bool packed_rows(PyObject *o, int64_t tokens, int64_t heads, int64_t D, sta_head_rows &r)
{
    if (!THPVariable_CheckExact(o)) return false;
    const at::Tensor &t = THPVariable_Unpack(o);
    if (!t.is_cuda() || t.layout() != at::kStrided || t.dim() != 3 || t.numel() == 0 || t.scalar_type() != at::kBFloat16) return false;
    const auto size = t.sizes(), stride = t.strides();
    if (size[0] != tokens || size[1] != heads || size[2] != D || stride[2] != 1) return false;
    r = {t.data_ptr(), 0, stride[0], stride[1], (int)heads, kBf16};
    return true;
}
struct PackedShape {
    int64_t tq, Hq, tk, Hkv, D, S;
};
bool packed_shape(PyObject *q, PyObject *k, PyObject *cu_q, PackedShape &s)
{
    if (!THPVariable_CheckExact(q) || !THPVariable_CheckExact(k) || !THPVariable_CheckExact(cu_q)) return false;
    const at::Tensor &a = THPVariable_Unpack(q), &b = THPVariable_Unpack(k);
    if (a.dim() != 3 || b.dim() != 3) return false;
    s = {a.size(0), a.size(1), b.size(0), b.size(1), a.size(2), THPVariable_Unpack(cu_q).numel() - 1};
    return small(s.tq) && small(s.Hq) && small(s.tk) && small(s.Hkv) && small(s.D) && s.S >= 0 && small(s.S);
}
bool packed_lse(PyObject *o, const PackedShape &s, const void *&out)
{
    out = nullptr;
    if (o == Py_None) return true;
    View v;
    if (!dense(o, v) || v.t->dim() != 2 || v.t->size(0) != s.Hq || v.t->size(1) != s.tq || v.t->scalar_type() != at::kFloat) return false;
    out = v.ptr;
    return out != nullptr;
}

// (q, k, v, o, cu_q, cu_k, max_q, max_k, causal, scale, lse, k_used, workspace)
PyObject *py_packed_forward(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    return guarded([&]() -> PyObject * {
        PackedShape s;
        sta_head_rows r[4];
        const void *cu_q, *cu_k, *used, *lse;
        int max_q, max_k;
        float scale;
        void *ws, *stream;
        size_t bytes;
        if (!layers.packed_forward || n != 13 || !packed_shape(args[0], args[1], args[4], s) || !packed_rows(args[0], s.tq, s.Hq, s.D, r[0]) ||
            !packed_rows(args[1], s.tk, s.Hkv, s.D, r[1]) || !packed_rows(args[2], s.tk, s.Hkv, s.D, r[2]) || !packed_rows(args[3], s.tq, s.Hq, s.D, r[3]) ||
            args[4] == Py_None || args[5] == Py_None || !vector(args[4], s.S + 1, at::kInt, cu_q) || !vector(args[5], s.S + 1, at::kInt, cu_k) ||
            !integer(args[6], max_q) || !integer(args[7], max_k) || !PyBool_Check(args[8]) || !number(args[9], scale) || !packed_lse(args[10], s, lse) ||
            !vector(args[11], s.S, at::kInt, used) || !scratch(args[12], ws, bytes))
            Py_RETURN_NONE;
        if (!stream_of(stream)) return nullptr;
        return status_of([&]() {
            return layers.packed_forward(&r[0], &r[1], &r[2], &r[3], static_cast<float *>(const_cast<void *>(lse)), s.tq, s.tk,
                                         static_cast<const int32_t *>(cu_q), static_cast<const int32_t *>(cu_k), static_cast<const int32_t *>(used),
                                         (int)s.S, max_q, max_k, (int)s.D, args[8] == Py_True, scale, ws, bytes, stream);
        });
    });
}

// (q, k, v, o, d_o, lse, d_q, d_k, d_v, cu_q, cu_k, max_q, max_k, workspace, causal, scale)
PyObject *py_packed_backward(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    return guarded([&]() -> PyObject * {
        PackedShape s;
        sta_head_rows r[8];
        const void *cu_q, *cu_k, *lse;
        int max_q, max_k;
        float scale;
        void *ws, *stream;
        size_t bytes;
        if (!layers.packed_backward || n != 16 || !packed_shape(args[0], args[1], args[9], s) || args[5] == Py_None || !packed_lse(args[5], s, lse) ||
            args[9] == Py_None || args[10] == Py_None || !vector(args[9], s.S + 1, at::kInt, cu_q) || !vector(args[10], s.S + 1, at::kInt, cu_k) ||
            !integer(args[11], max_q) || !integer(args[12], max_k) || !scratch(args[13], ws, bytes) || !PyBool_Check(args[14]) || !number(args[15], scale))
            Py_RETURN_NONE;
        for (int i = 0; i < 8; ++i) {                       // q k v o d_o d_q d_k d_v
            const bool keys = i == 1 || i == 2 || i >= 6;
            if (!packed_rows(args[i < 5 ? i : i + 1], keys ? s.tk : s.tq, keys ? s.Hkv : s.Hq, s.D, r[i])) Py_RETURN_NONE;
        }
        if (!stream_of(stream)) return nullptr;
        return status_of([&]() {
            return layers.packed_backward(&r[0], &r[1], &r[2], &r[3], &r[4], static_cast<const float *>(lse), &r[5], &r[6], &r[7], s.tq, s.tk,
                                          static_cast<const int32_t *>(cu_q), static_cast<const int32_t *>(cu_k), (int)s.S, max_q, max_k, (int)s.D,
                                          args[14] == Py_True, scale, ws, bytes, stream);
        });
    });
}

// (addresses of the five entry points in the order of LayerEntries); the streams are bind's
PyObject *py_bind_layers(PyObject *, PyObject *args)
{
    unsigned long long a[5];
    if (!PyArg_ParseTuple(args, "KKKKK", &a[0], &a[1], &a[2], &a[3], &a[4])) return nullptr;
    if (current_device && current_raw_stream)
        layers = {reinterpret_cast<decltype(&sta_rope)>(a[0]), reinterpret_cast<decltype(&sta_qk_norm_rope)>(a[1]),
                  reinterpret_cast<decltype(&sta_qk_norm_rope_backward)>(a[2]), reinterpret_cast<decltype(&sta_packed_forward)>(a[3]),
                  reinterpret_cast<decltype(&sta_packed_backward)>(a[4])};
    Py_RETURN_NONE;
}

// (addresses of the five entry points in the order of Entries, torch's current device and raw current stream)
PyObject *py_bind(PyObject *, PyObject *args)
{
    unsigned long long a[5];
    PyObject *device, *stream;
    if (!PyArg_ParseTuple(args, "KKKKKOO", &a[0], &a[1], &a[2], &a[3], &a[4], &device, &stream)) return nullptr;
    Py_INCREF(device);
    Py_INCREF(stream);
    Py_XSETREF(current_device, device);
    Py_XSETREF(current_raw_stream, stream);
    entries.tile_permute = reinterpret_cast<PermuteFn>(a[0]);
    entries.untile = reinterpret_cast<PermuteFn>(a[1]);
    entries.forward = reinterpret_cast<ForwardFn>(a[2]);
    entries.forward_lse = reinterpret_cast<ForwardLseFn>(a[3]);
    entries.backward = reinterpret_cast<BackwardFn>(a[4]);
    Py_RETURN_NONE;
}

#define STA_FAST(name) {#name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(py_##name)), METH_FASTCALL, nullptr}
PyMethodDef methods[] = {
    {"bind", py_bind, METH_VARARGS, nullptr}, STA_FAST(tile_permute), STA_FAST(untile), STA_FAST(forward), STA_FAST(forward_lse),
    STA_FAST(backward), {"bind_layers", py_bind_layers, METH_VARARGS, nullptr}, STA_FAST(rope), STA_FAST(norm_rope), STA_FAST(norm_rope_backward),
    STA_FAST(packed_forward), STA_FAST(packed_backward), {nullptr, nullptr, 0, nullptr},
};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "sta_fastcall", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit_sta_fastcall(void) { return PyModule_Create(&module); }
