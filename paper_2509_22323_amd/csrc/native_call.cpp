// The entry points that launch, called with tensors: checks and marshalling of binding.py in native code.  A call of few tokens
// costs what the host needs to issue it.  us of host time a call by way of ctypes / here, and on the GPU in a graph, H = 2, N = 256,
// D = 64: dense 5.9 / 3.0, 4.2; block-sparse 7.2 / 3.2, 5.6; joint, two segments 11.0 / 3.2, 4.6; selection (two launches) 9.2 / 5.6, 5.0.
//
// Every function returns the library's status, or None for arguments that are not what most calls hand over (subclasses of
// Tensor, tensors without storage, shapes that do not fit, numbers of other types, no workspace): binding.py then goes its own
// way, which has every check and every message.  Nothing is kept from one call for the next.
#define PY_SSIZE_T_CLEAN
#include <Python.h>
#include <limits.h>
#include <string.h>

#include <c10/core/impl/DeviceGuardImplInterface.h>
#include <torch/csrc/autograd/python_variable.h>

#include "rapid_attn.h"
#include "rapid_cache.h"
#include "rapid_layer.h"
#include "rapid_mask.h"
#include "rapid_packed.h"

namespace {

PyObject* current_stream = nullptr;                // torch._C._cuda_getCurrentRawStream
PyObject* axis_type = nullptr;                     // RopeAxis of binding.py, a rapid_rope_axis in a buffer

decltype(&rapid_attn_dense) attn_dense;
decltype(&rapid_attn_block_sparse) attn_block_sparse;
decltype(&rapid_attn_joint) attn_joint;
decltype(&rapid_attn_joint_select) attn_joint_select;
decltype(&rapid_mask_select) mask_select;
decltype(&rapid_cache_store) cache_store;
decltype(&rapid_cache_reuse) cache_reuse;
decltype(&rapid_linear) layer_linear;
decltype(&rapid_linear_workspace_bytes) layer_linear_bytes;
decltype(&rapid_norm_modulate) layer_modulate;
decltype(&rapid_rope_table) layer_table;
decltype(&rapid_qk_norm_rope) layer_qk;
decltype(&rapid_rope) layer_rope;
decltype(&rapid_quantize_rows) rows_quantize;
decltype(&rapid_norm_modulate_int8) rows_modulate;
decltype(&rapid_linear_int8) int8_linear;
decltype(&rapid_linear_int8_workspace_bytes) int8_linear_bytes;
decltype(&rapid_attn_packed) attn_packed;

// A tensor of exactly that class with memory of its own on a GPU; else null.
const at::Tensor* plain(PyObject* o)
{
    if (!THPVariable_CheckExact(o)) return nullptr;
    const at::Tensor& t = THPVariable_Unpack(o);
    if (!t.defined() || !t.has_storage() || t.layout() != at::kStrided || !t.is_cuda()) return nullptr;
    return &t;
}
const at::Tensor* of(PyObject* o, at::ScalarType type)
{
    const at::Tensor* t = plain(o);
    return t && t->scalar_type() == type ? t : nullptr;
}
// Contiguous, on a device, of a type.
const at::Tensor* packed(PyObject* o, at::ScalarType type, int device)
{
    const at::Tensor* t = of(o, type);
    return t && t->is_contiguous() && t->get_device() == device ? t : nullptr;
}

bool integer(PyObject* o, int& v)
{
    if (!PyLong_CheckExact(o)) return false;
    int over = 0;
    const long long x = PyLong_AsLongLongAndOverflow(o, &over);
    if (over || x < INT_MIN || x > INT_MAX) return false;
    v = (int)x;
    return true;
}
bool number(PyObject* o, double& v)
{
    if (PyFloat_CheckExact(o)) { v = PyFloat_AS_DOUBLE(o); return true; }
    int i;
    if (!integer(o, i)) return false;
    v = i;
    return true;
}
bool number(PyObject* o, float& v)
{
    double d;
    if (!number(o, d)) return false;
    v = (float)d;
    return true;
}
bool size(int64_t n, int& v)
{
    if (n < 0 || n > INT_MAX) return false;
    v = (int)n;
    return true;
}

// torch's current stream on the device; false: an exception is set
bool stream_on(int device, void*& stream)
{
    PyObject* d = PyLong_FromLong(device);
    if (!d) return false;
    PyObject* s = PyObject_CallOneArg(current_stream, d);
    Py_DECREF(d);
    if (!s) return false;
    stream = PyLong_AsVoidPtr(s);
    Py_DECREF(s);
    return !(stream == nullptr && PyErr_Occurred());
}

// The call itself, without the interpreter's lock (as ctypes makes it).
template <class Call>
PyObject* launch(int device, Call call)
{
    void* stream;
    if (!stream_on(device, stream)) return nullptr;
    int status;
    Py_BEGIN_ALLOW_THREADS
    status = call(stream);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(status);
}

// q, k, v, o (or q, k alone) contiguous [B, H, N, D]
struct Bhnd {
    const at::Tensor* t[4];
    int B, H, N, D, device;
};
bool bhnd(PyObject* const* a, int n, Bhnd& x)
{
    for (int i = 0; i < n; ++i) {
        const at::Tensor* t = of(a[i], at::kBFloat16);
        if (!t || t->dim() != 4 || !t->is_contiguous()) return false;
        if (i == 0) {
            x.device = t->get_device();
            if (!size(t->size(0), x.B) || !size(t->size(1), x.H) || !size(t->size(2), x.N) || !size(t->size(3), x.D)) return false;
        } else if (t->sizes() != x.t[0]->sizes() || t->get_device() != x.device) return false;
        x.t[i] = t;
    }
    return true;
}
bool length(PyObject* o, int none, int& v)
{
    if (o == Py_None) { v = none; return true; }
    return integer(o, v);
}
bool is_grid(const at::Tensor& mask, int B, int H, int nb)
{
    return mask.dim() == 4 && mask.size(0) == B && mask.size(1) == H && mask.size(2) == nb && mask.size(3) == nb;
}

// (q, k, v, o, kv_len, scale)
PyObject* dense(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    Bhnd x;
    int kv_len;
    float scale;
    if (n != 6 || !bhnd(a, 4, x) || !length(a[4], x.N, kv_len) || !number(a[5], scale)) Py_RETURN_NONE;
    void *q = x.t[0]->data_ptr(), *k = x.t[1]->data_ptr(), *v = x.t[2]->data_ptr(), *o = x.t[3]->data_ptr();
    return launch(x.device, [&](void* s) { return attn_dense(q, k, v, o, x.B, x.H, x.N, x.D, kv_len, scale, nullptr, 0, s); });
}

// (q, k, v, o, mask, block, kv_len, scale, workspace)
PyObject* block_sparse(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    Bhnd x;
    int block, kv_len;
    float scale;
    if (n != 9 || !bhnd(a, 4, x) || !integer(a[5], block) || !length(a[6], x.N, kv_len) || !number(a[7], scale)) Py_RETURN_NONE;
    const at::Tensor *mask = packed(a[4], at::kByte, x.device), *ws = plain(a[8]);
    if (!mask || block <= 0 || x.N % block != 0 || !is_grid(*mask, x.B, x.H, x.N / block)) Py_RETURN_NONE;
    if (!ws || !ws->is_contiguous() || ws->get_device() != x.device) Py_RETURN_NONE;
    void *q = x.t[0]->data_ptr(), *k = x.t[1]->data_ptr(), *v = x.t[2]->data_ptr(), *o = x.t[3]->data_ptr();
    const auto* m = (const unsigned char*)mask->data_ptr();
    void* w = ws->data_ptr();
    const size_t bytes = ws->nbytes();
    return launch(x.device, [&](void* s) {
        return attn_block_sparse(q, k, v, o, x.B, x.H, x.N, x.D, block, m, kv_len, scale, w, bytes, s);
    });
}

// (q, k, mask, block, kv_len, text_start, tau, scale, workspace)
PyObject* select(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    Bhnd x;
    int block, kv_len, text_start;
    float tau, scale;
    if (n != 9 || !bhnd(a, 2, x) || !integer(a[3], block) || !length(a[4], x.N, kv_len) || !length(a[5], x.N, text_start)) Py_RETURN_NONE;
    if (!number(a[6], tau) || !number(a[7], scale)) Py_RETURN_NONE;
    const at::Tensor *mask = packed(a[2], at::kByte, x.device), *ws = plain(a[8]);
    if (!mask || block <= 0 || x.N % block != 0 || !is_grid(*mask, x.B, x.H, x.N / block) || !ws) Py_RETURN_NONE;
    void *q = x.t[0]->data_ptr(), *k = x.t[1]->data_ptr(), *w = ws->data_ptr();
    auto* m = (unsigned char*)mask->data_ptr();
    const size_t bytes = ws->nbytes();
    return launch(x.device, [&](void* s) {
        return mask_select(q, k, x.B, x.H, x.N, x.D, block, kv_len, text_start, tau, scale, m, w, bytes, s);
    });
}

// One or two (q, k, v, o) of [B, H, n, D] with strides.
struct Joint {
    rapid_attn_segment seg[2];
    int n, B, H, N, D, device;
};
bool joint_segments(PyObject* list, Joint& x)
{
    if (!PyList_CheckExact(list) && !PyTuple_CheckExact(list)) return false;
    const Py_ssize_t n = PySequence_Fast_GET_SIZE(list);
    if (n != 1 && n != 2) return false;
    x.n = (int)n;
    int64_t tokens = 0;
    for (Py_ssize_t i = 0; i < n; ++i) {
        PyObject* one = PySequence_Fast_GET_ITEM(list, i);
        if ((!PyList_CheckExact(one) && !PyTuple_CheckExact(one)) || PySequence_Fast_GET_SIZE(one) != 4) return false;
        const at::Tensor* t[4];
        for (int j = 0; j < 4; ++j) {
            t[j] = of(PySequence_Fast_GET_ITEM(one, j), at::kBFloat16);
            if (!t[j] || t[j]->dim() != 4 || t[j]->stride(3) != 1) return false;
            if (j > 0 && (t[j]->sizes() != t[0]->sizes() || t[j]->get_device() != t[0]->get_device())) return false;
            if ((j == 1 || j == 2) && t[j]->strides() != t[0]->strides()) return false;
        }
        int B, H, D;
        rapid_attn_segment& g = x.seg[i];
        if (!size(t[0]->size(0), B) || !size(t[0]->size(1), H) || !size(t[0]->size(2), g.n) || !size(t[0]->size(3), D)) return false;
        if (i == 0) { x.B = B; x.H = H; x.D = D; x.device = t[0]->get_device(); }
        else if (B != x.B || H != x.H || D != x.D) return false;
        g.q = t[0]->data_ptr(); g.k = t[1]->data_ptr(); g.v = t[2]->data_ptr(); g.o = t[3]->data_ptr();
        g.in_stride_b = t[0]->stride(0); g.in_stride_h = t[0]->stride(1); g.in_stride_n = t[0]->stride(2);
        g.out_stride_b = t[3]->stride(0); g.out_stride_h = t[3]->stride(1); g.out_stride_n = t[3]->stride(2);
        tokens += g.n;
    }
    return size(tokens, x.N);
}
bool lengths(PyObject* o, const Joint& x, const int*& p)
{
    p = nullptr;
    if (o == Py_None) return true;
    const at::Tensor* t = packed(o, at::kInt, x.device);
    if (!t || t->numel() != x.B) return false;
    p = (const int*)t->data_ptr();
    return true;
}
inline int blocks(int N, int block) { return block > 0 ? (int)(((long long)N + block - 1) / block) : 0; }

// (segments, mask or None, block, kv_len, kv_lens, scale, workspace)
PyObject* joint(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    Joint x;
    int block, kv_len;
    float scale;
    const int* lens;
    if (n != 7 || !joint_segments(a[0], x) || !integer(a[2], block) || !length(a[3], 0, kv_len) || !lengths(a[4], x, lens)) Py_RETURN_NONE;
    if (!number(a[5], scale)) Py_RETURN_NONE;
    const unsigned char* m = nullptr;
    void* w = nullptr;
    size_t bytes = 0;
    if (a[1] != Py_None) {
        const at::Tensor *mask = packed(a[1], at::kByte, x.device), *ws = plain(a[6]);
        if (!mask || !ws || !is_grid(*mask, x.B, x.H, blocks(x.N, block))) Py_RETURN_NONE;
        m = (const unsigned char*)mask->data_ptr();
        w = ws->data_ptr();
        bytes = ws->nbytes();
    }
    return launch(x.device, [&](void* s) {
        return attn_joint(x.seg, x.n, x.B, x.H, x.D, block, m, kv_len, lens, scale, w, bytes, s);
    });
}

// (segments, block, kv_len, kv_lens, text_start, tau, scale, mask_out or None, workspace)
PyObject* joint_select(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    Joint x;
    int block, kv_len, text_start;
    float tau, scale;
    const int* lens;
    if (n != 9 || !joint_segments(a[0], x) || !integer(a[1], block) || !length(a[2], 0, kv_len) || !lengths(a[3], x, lens)) Py_RETURN_NONE;
    if (!length(a[4], x.N, text_start) || !number(a[5], tau) || !number(a[6], scale)) Py_RETURN_NONE;
    const at::Tensor* ws = plain(a[8]);
    if (!ws) Py_RETURN_NONE;
    unsigned char* m = nullptr;
    if (a[7] != Py_None) {
        const at::Tensor* mask = packed(a[7], at::kByte, x.device);
        if (!mask || !is_grid(*mask, x.B, x.H, blocks(x.N, block))) Py_RETURN_NONE;
        m = (unsigned char*)mask->data_ptr();
    }
    void* w = ws->data_ptr();
    const size_t bytes = ws->nbytes();
    return launch(x.device, [&](void* s) {
        return attn_joint_select(x.seg, x.n, x.B, x.H, x.D, block, kv_len, lens, text_start, tau, scale, m, w, bytes, s);
    });
}

// (a, b, out, flags or None)
template <class Call>
PyObject* residual(PyObject* const* a, Py_ssize_t n, Call call)
{
    if (n != 4) Py_RETURN_NONE;
    const at::Tensor* t[3];
    for (int i = 0; i < 3; ++i) {
        t[i] = of(a[i], at::kBFloat16);
        if (!t[i] || !t[i]->is_contiguous() || t[i]->dim() < 1) Py_RETURN_NONE;
        if (i > 0 && (t[i]->sizes() != t[0]->sizes() || t[i]->get_device() != t[0]->get_device())) Py_RETURN_NONE;
    }
    int B;
    if (!size(t[0]->size(0), B)) Py_RETURN_NONE;
    const size_t per = B > 0 ? (size_t)(t[0]->numel() / B) : 0;
    const int device = t[0]->get_device();
    const unsigned char* flags = nullptr;
    if (a[3] != Py_None) {
        const at::Tensor* f = packed(a[3], at::kByte, device);
        if (!f || f->numel() != B) Py_RETURN_NONE;
        flags = (const unsigned char*)f->data_ptr();
    }
    void *x = t[0]->data_ptr(), *y = t[1]->data_ptr(), *out = t[2]->data_ptr();
    return launch(device, [&](void* s) { return call(x, y, out, B, per, flags, s); });
}
PyObject* store(PyObject*, PyObject* const* a, Py_ssize_t n) { return residual(a, n, cache_store); }
PyObject* reuse(PyObject*, PyObject* const* a, Py_ssize_t n) { return residual(a, n, cache_reuse); }

// ---- a layer around its attention: tensors of the current device alone (the Python form makes another one current)
bool current(int device) { return c10::impl::getDeviceGuardImpl(at::kCUDA)->getDevice().index() == device; }

// [B, n, width] or [n, width] with a contiguous last dimension
struct Rows3 {
    rapid_rows rows;
    int B, n, width, device;
};
bool rows3(PyObject* o, Rows3& x, at::ScalarType type = at::kBFloat16)
{
    const at::Tensor* t = of(o, type);
    if (!t || (t->dim() != 2 && t->dim() != 3)) return false;
    const int d = (int)t->dim();
    x.B = 1;
    if ((d == 3 && !size(t->size(0), x.B)) || !size(t->size(d - 2), x.n) || !size(t->size(d - 1), x.width)) return false;
    if (t->stride(d - 1) != 1 && x.width != 1) return false;
    x.rows = {t->data_ptr(), d == 3 ? t->stride(0) : 0, t->stride(d - 2)};
    x.device = t->get_device();
    return true;
}
// None, or [B, width] or [width] with a contiguous last dimension
bool vectors(PyObject* o, const Rows3& like, const void*& p, long long& stride)
{
    p = nullptr;
    stride = 0;
    if (o == Py_None) return true;
    const at::Tensor* t = of(o, at::kBFloat16);
    if (!t || (t->dim() != 1 && t->dim() != 2) || t->get_device() != like.device) return false;
    const int d = (int)t->dim();
    if (t->size(d - 1) != like.width || (t->stride(d - 1) != 1 && like.width != 1)) return false;
    if (d == 2) {
        if (t->size(0) != like.B) return false;
        stride = t->stride(0);
    }
    p = t->data_ptr();
    return true;
}
bool is(PyObject* o, const char* text) { return PyUnicode_CheckExact(o) && PyUnicode_CompareWithASCIIString(o, text) == 0; }

// (x, weight, out, bias, activation, gate, residual, workspace or None where none is made use of)
PyObject* linear(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    Rows3 x, out, res;
    if (n != 8 || !rows3(a[0], x) || !rows3(a[2], out) || out.B != x.B || out.n != x.n || out.device != x.device || !current(x.device)) Py_RETURN_NONE;
    const at::Tensor* w = of(a[1], at::kBFloat16);
    if (!w || w->dim() != 2 || w->size(0) != out.width || w->size(1) != x.width || w->get_device() != x.device) Py_RETURN_NONE;
    if (w->stride(1) != 1 && x.width != 1) Py_RETURN_NONE;
    const void *bias, *gate;
    long long unused, gate_stride;
    if (!vectors(a[3], out, bias, unused) || (bias && THPVariable_Unpack(a[3]).dim() != 1) || !vectors(a[5], out, gate, gate_stride)) Py_RETURN_NONE;
    const int activation = is(a[4], "none") ? RAPID_ACT_NONE : is(a[4], "silu") ? RAPID_ACT_SILU : is(a[4], "gelu_tanh") ? RAPID_ACT_GELU_TANH : -1;
    if (activation < 0) Py_RETURN_NONE;
    if (a[6] != Py_None && (!rows3(a[6], res) || res.B != out.B || res.n != out.n || res.width != out.width || res.device != x.device)) Py_RETURN_NONE;
    void* ws = nullptr;
    size_t bytes = 0;
    if (a[7] != Py_None) {
        const at::Tensor* t = plain(a[7]);
        if (!t || !t->is_contiguous() || t->get_device() != x.device) Py_RETURN_NONE;
        ws = t->data_ptr();
        bytes = t->nbytes();
    } else if (layer_linear_bytes((long long)x.B * x.n, out.width, x.width) != 0) Py_RETURN_NONE;
    const void* weight = w->data_ptr();
    const long long w_stride = out.width > 1 ? w->stride(0) : x.width;
    const rapid_rows* residual = a[6] != Py_None ? &res.rows : nullptr;
    return launch(x.device, [&](void* s) {
        return layer_linear(&x.rows, weight, w_stride, bias, &out.rows, activation, gate, gate_stride, residual, x.B, x.n, out.width, x.width,
                            ws, bytes, s);
    });
}

// (x, out, scale, shift, eps)
PyObject* modulate(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    Rows3 x, out;
    float eps;
    const void *scale, *shift;
    long long scale_stride, shift_stride;
    if (n != 5 || !rows3(a[0], x) || !rows3(a[1], out) || out.B != x.B || out.n != x.n || out.width != x.width || out.device != x.device) Py_RETURN_NONE;
    if (!current(x.device) || !vectors(a[2], x, scale, scale_stride) || !vectors(a[3], x, shift, shift_stride) || !scale != !shift) Py_RETURN_NONE;
    if (!number(a[4], eps)) Py_RETURN_NONE;
    return launch(x.device, [&](void* s) {
        return layer_modulate(&x.rows, &out.rows, scale, scale_stride, shift, shift_stride, x.B, x.n, x.width, eps, s);
    });
}

// (positions, axes: a list or tuple of RopeAxis, table, magnitude)
PyObject* table(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    if (n != 4 || (!PyList_CheckExact(a[1]) && !PyTuple_CheckExact(a[1]))) Py_RETURN_NONE;
    const at::Tensor *p = of(a[0], at::kInt), *t = of(a[2], at::kFloat);
    const Py_ssize_t axes = PySequence_Fast_GET_SIZE(a[1]);
    double magnitude;
    if (!p || !t || axes < 1 || axes > 8 || !p->is_contiguous() || !t->is_contiguous() || t->get_device() != p->get_device()) Py_RETURN_NONE;
    if (!current(p->get_device()) || p->dim() < 2 || t->dim() != p->dim() + 1 || p->size(-1) != axes || t->size(-1) != 2) Py_RETURN_NONE;
    if (p->sizes().slice(0, p->dim() - 1) != t->sizes().slice(0, t->dim() - 2) || !number(a[3], magnitude)) Py_RETURN_NONE;
    rapid_rope_axis axis[8];
    int64_t dims = 0;
    for (Py_ssize_t i = 0; i < axes; ++i) {
        Py_buffer b;
        PyObject* o = PySequence_Fast_GET_ITEM(a[1], i);
        if (!PyType_IsSubtype(Py_TYPE(o), (PyTypeObject*)axis_type)) Py_RETURN_NONE;
        if (PyObject_GetBuffer(o, &b, PyBUF_SIMPLE) != 0) { PyErr_Clear(); Py_RETURN_NONE; }
        const bool fits = b.len == (Py_ssize_t)sizeof(rapid_rope_axis);
        if (fits) memcpy(&axis[i], b.buf, sizeof(rapid_rope_axis));
        PyBuffer_Release(&b);
        if (!fits) Py_RETURN_NONE;
        dims += axis[i].dim;
    }
    if (dims != 2 * t->size(-2)) Py_RETURN_NONE;
    const int* positions = (const int*)p->data_ptr();
    float* out = (float*)t->data_ptr();
    const long long tokens = p->numel() / axes;
    return launch(p->get_device(), [&](void* s) { return layer_table(positions, tokens, (int)axes, axis, magnitude, out, s); });
}

// (segments of (q, k, q_out, k_out), weights or None, table or None, layout): both forms
struct QkCall {
    rapid_qk_segment seg[2];
    int n, B, H, D, device, rot, layout;
    const float* table;
    long long table_stride;
};
bool qk_call(PyObject* const* a, QkCall& x)
{
    if (!PyList_CheckExact(a[0]) && !PyTuple_CheckExact(a[0])) return false;
    const Py_ssize_t n = PySequence_Fast_GET_SIZE(a[0]);
    const bool weighted = a[1] != Py_None;
    if (n != 1 && n != 2) return false;
    if (weighted && ((!PyList_CheckExact(a[1]) && !PyTuple_CheckExact(a[1])) || PySequence_Fast_GET_SIZE(a[1]) != n)) return false;
    int64_t tokens = 0;
    x.n = (int)n;
    for (Py_ssize_t i = 0; i < n; ++i) {
        PyObject* one = PySequence_Fast_GET_ITEM(a[0], i);
        if ((!PyList_CheckExact(one) && !PyTuple_CheckExact(one)) || PySequence_Fast_GET_SIZE(one) != 4) return false;
        const at::Tensor* t[4];
        for (int j = 0; j < 4; ++j) {
            t[j] = of(PySequence_Fast_GET_ITEM(one, j), at::kBFloat16);
            if (!t[j] || t[j]->dim() != 4 || t[j]->stride(3) != 1) return false;
            if (j > 0 && (t[j]->sizes() != t[0]->sizes() || t[j]->get_device() != t[0]->get_device())) return false;
        }
        if (t[1]->strides() != t[0]->strides() || t[3]->strides() != t[2]->strides()) return false;
        int B, H, D;
        rapid_qk_segment& g = x.seg[i];
        g = {};
        if (!size(t[0]->size(0), B) || !size(t[0]->size(1), H) || !size(t[0]->size(2), g.n) || !size(t[0]->size(3), D)) return false;
        if (i == 0) { x.B = B; x.H = H; x.D = D; x.device = t[0]->get_device(); }
        else if (B != x.B || H != x.H || D != x.D || t[0]->get_device() != x.device) return false;
        g.q = t[0]->data_ptr(); g.k = t[1]->data_ptr(); g.q_out = t[2]->data_ptr(); g.k_out = t[3]->data_ptr();
        g.in_stride_b = t[0]->stride(0); g.in_stride_h = t[0]->stride(1); g.in_stride_n = t[0]->stride(2);
        g.out_stride_b = t[2]->stride(0); g.out_stride_h = t[2]->stride(1); g.out_stride_n = t[2]->stride(2);
        if (weighted) {
            PyObject* two = PySequence_Fast_GET_ITEM(a[1], i);
            if ((!PyList_CheckExact(two) && !PyTuple_CheckExact(two)) || PySequence_Fast_GET_SIZE(two) != 2) return false;
            const void** to[2] = {&g.q_weight, &g.k_weight};
            for (int j = 0; j < 2; ++j) {
                PyObject* w = PySequence_Fast_GET_ITEM(two, j);
                if (w == Py_None) continue;
                const at::Tensor* v = packed(w, at::kBFloat16, x.device);
                if (!v || v->dim() != 1 || v->size(0) != D) return false;
                *to[j] = v->data_ptr();
            }
        }
        tokens += g.n;
    }
    x.layout = is(a[3], "interleaved") ? RAPID_ROPE_INTERLEAVED : is(a[3], "half") ? RAPID_ROPE_HALVES : -1;
    x.table = nullptr;
    x.table_stride = 0;
    x.rot = 0;
    if (x.layout < 0 || !current(x.device)) return false;
    if (a[2] == Py_None) return true;
    const at::Tensor* t = packed(a[2], at::kFloat, x.device);
    if (!t || (t->dim() != 3 && t->dim() != 4) || t->size(-1) != 2 || t->size(-3) != tokens || t->size(-2) > 64) return false;
    if (t->dim() == 4) {
        if (t->size(0) != x.B) return false;
        x.table_stride = t->stride(0);
    }
    x.rot = 2 * (int)t->size(-2);
    x.table = (const float*)t->data_ptr();
    return true;
}

// (segments, weights, table, layout, eps)
PyObject* qk_norm_rope(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    QkCall x;
    float eps;
    if (n != 5 || !qk_call(a, x) || !number(a[4], eps)) Py_RETURN_NONE;
    return launch(x.device, [&](void* s) { return layer_qk(x.seg, x.n, x.B, x.H, x.D, eps, x.table, x.table_stride, x.rot, x.layout, s); });
}

// (segments, None, table, layout)
PyObject* rope(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    QkCall x;
    if (n != 4 || a[1] != Py_None || a[2] == Py_None || !qk_call(a, x)) Py_RETURN_NONE;
    return launch(x.device, [&](void* s) { return layer_rope(x.seg, x.n, x.B, x.H, x.D, x.table, x.table_stride, x.rot, x.layout, s); });
}

// ---- layers in 8 bits over packed sequences
// None, or a contiguous tensor [B, n], or [n] where B is 1
bool per_row(PyObject* o, at::ScalarType type, const Rows3& like, const void*& p)
{
    p = nullptr;
    if (o == Py_None) return true;
    const at::Tensor* t = packed(o, type, like.device);
    if (!t) return false;
    if (t->dim() == 2 ? t->size(0) != like.B || t->size(1) != like.n : t->dim() != 1 || like.B != 1 || t->size(0) != like.n) return false;
    p = t->data_ptr();
    return true;
}
// Rows of the conditioning's vectors: the samples, or the documents that vectors of two dimensions have (they have to agree), or any number.
bool vector_rows(PyObject* const* a, int n, bool documents, const Rows3& like, Rows3& rows)
{
    rows = like;
    if (!documents) return true;
    rows.B = INT_MAX;
    for (int i = 0; i < n; ++i) {
        if (a[i] == Py_None) continue;
        const at::Tensor* t = plain(a[i]);
        int count;
        if (!t) return false;
        if (t->dim() != 2) continue;
        if (!size(t->size(0), count) || (rows.B != INT_MAX && rows.B != count)) return false;
        rows.B = count;
    }
    return true;
}

// (x, q, scale)
PyObject* quantize(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    Rows3 x, q;
    const void* scale;
    if (n != 3 || !rows3(a[0], x) || !rows3(a[1], q, at::kChar) || q.B != x.B || q.n != x.n || q.width != x.width || q.device != x.device) Py_RETURN_NONE;
    if (!current(x.device) || a[2] == Py_None || !per_row(a[2], at::kFloat, x, scale)) Py_RETURN_NONE;
    return launch(x.device, [&](void* s) { return rows_quantize(&x.rows, &q.rows, (float*)scale, x.B, x.n, x.width, s); });
}

// (x, q, q_scale, scale, shift, eps, document)
PyObject* modulate8(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    Rows3 x, q, rows;
    const void *q_scale, *scale, *shift, *document;
    long long scale_stride, shift_stride;
    float eps;
    if (n != 7 || !rows3(a[0], x) || !rows3(a[1], q, at::kChar) || q.B != x.B || q.n != x.n || q.width != x.width || q.device != x.device) Py_RETURN_NONE;
    if (!current(x.device) || a[2] == Py_None || !per_row(a[2], at::kFloat, x, q_scale) || !per_row(a[6], at::kInt, x, document)) Py_RETURN_NONE;
    if (!vector_rows(a + 3, 2, document != nullptr, x, rows) || !vectors(a[3], rows, scale, scale_stride) || !vectors(a[4], rows, shift, shift_stride)) Py_RETURN_NONE;
    if (!scale != !shift || !number(a[5], eps)) Py_RETURN_NONE;
    return launch(x.device, [&](void* s) {
        return rows_modulate(&x.rows, &q.rows, (float*)q_scale, scale, scale_stride, shift, shift_stride, (const int*)document, document ? rows.B : 0,
                             x.B, x.n, x.width, eps, s);
    });
}

// (x, x_scale, weight, w_scale, out, bias, activation, gate, residual, document, workspace or None where none is made use of)
PyObject* linear8(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    Rows3 x, out, res, rows;
    if (n != 11 || !rows3(a[0], x, at::kChar) || !rows3(a[4], out) || out.B != x.B || out.n != x.n || out.device != x.device || !current(x.device)) Py_RETURN_NONE;
    const at::Tensor *w = of(a[2], at::kChar), *ws_scale = packed(a[3], at::kFloat, x.device);
    if (!w || w->dim() != 2 || w->size(0) != out.width || w->size(1) != x.width || w->get_device() != x.device) Py_RETURN_NONE;
    if ((w->stride(1) != 1 && x.width != 1) || !ws_scale || ws_scale->dim() != 1 || ws_scale->size(0) != out.width) Py_RETURN_NONE;
    const void *x_scale, *document, *bias, *gate;
    long long unused, gate_stride;
    if (a[1] == Py_None || !per_row(a[1], at::kFloat, x, x_scale) || !per_row(a[9], at::kInt, x, document)) Py_RETURN_NONE;
    if (!vectors(a[5], out, bias, unused) || (bias && THPVariable_Unpack(a[5]).dim() != 1)) Py_RETURN_NONE;
    if (!vector_rows(a + 7, 1, document != nullptr, out, rows) || !vectors(a[7], rows, gate, gate_stride)) Py_RETURN_NONE;
    const int activation = is(a[6], "none") ? RAPID_ACT_NONE : is(a[6], "silu") ? RAPID_ACT_SILU : is(a[6], "gelu_tanh") ? RAPID_ACT_GELU_TANH : -1;
    if (activation < 0) Py_RETURN_NONE;
    if (a[8] != Py_None && (!rows3(a[8], res) || res.B != out.B || res.n != out.n || res.width != out.width || res.device != x.device)) Py_RETURN_NONE;
    void* ws = nullptr;
    size_t bytes = 0;
    if (a[10] != Py_None) {
        const at::Tensor* t = plain(a[10]);
        if (!t || !t->is_contiguous() || t->get_device() != x.device) Py_RETURN_NONE;
        ws = t->data_ptr();
        bytes = t->nbytes();
    } else if (int8_linear_bytes((long long)x.B * x.n, out.width, x.width) != 0) Py_RETURN_NONE;
    const void *weight = w->data_ptr(), *w_scale = ws_scale->data_ptr();
    const long long w_stride = out.width > 1 ? w->stride(0) : x.width;
    const rapid_rows* residual = a[8] != Py_None ? &res.rows : nullptr;
    return launch(x.device, [&](void* s) {
        return int8_linear(&x.rows, (const float*)x_scale, weight, w_stride, (const float*)w_scale, bias, &out.rows, activation, gate, gate_stride,
                           residual, (const int*)document, document ? rows.B : 0, x.B, x.n, out.width, x.width, ws, bytes, s);
    });
}

// int32 [B, N], or [N] (one for all samples), with a contiguous last dimension
bool per_token(PyObject* o, const Joint& x, const int*& p, long long& stride)
{
    const at::Tensor* t = of(o, at::kInt);
    if (!t || (t->dim() != 1 && t->dim() != 2) || t->get_device() != x.device) return false;
    const int d = (int)t->dim();
    if (t->size(d - 1) != x.N || (t->stride(d - 1) != 1 && x.N != 1) || (d == 2 && t->size(0) != x.B)) return false;
    p = (const int*)t->data_ptr();
    stride = d == 2 ? t->stride(0) : 0;
    return true;
}

// (segments, document, order or None, cap, scale, workspace)
PyObject* packed_attention(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    Joint x;
    const int *document, *order = nullptr;
    long long document_stride, order_stride = 0;
    float cap, scale;
    if (n != 6 || !joint_segments(a[0], x) || !current(x.device) || !number(a[3], cap) || !number(a[4], scale)) Py_RETURN_NONE;
    for (int i = 3; i < 5; ++i)                        // (more than 0, and 0 in fp32)
        if (double d; number(a[i], d) && d > 0.0 && (float)d == 0.f) Py_RETURN_NONE;
    for (int i = 0; i < x.n; ++i)                      // (segments of different devices)
        if (THPVariable_Unpack(PySequence_Fast_GET_ITEM(PySequence_Fast_GET_ITEM(a[0], i), 0)).get_device() != x.device) Py_RETURN_NONE;
    if (!per_token(a[1], x, document, document_stride) || (a[2] != Py_None && !per_token(a[2], x, order, order_stride))) Py_RETURN_NONE;
    const at::Tensor* t = plain(a[5]);
    if (!t || !t->is_contiguous() || t->get_device() != x.device) Py_RETURN_NONE;
    void* ws = t->data_ptr();
    const size_t bytes = t->nbytes();
    return launch(x.device, [&](void* s) {
        return attn_packed(x.seg, x.n, x.B, x.H, x.D, document, document_stride, order, order_stride, cap, scale, ws, bytes, s);
    });
}

// bind(address of each entry point, .., RopeAxis): of the library that binding.py has loaded
PyObject* bind(PyObject*, PyObject* args)
{
    unsigned long long p[18];
    PyTypeObject* axis;
    if (!PyArg_ParseTuple(args, "KKKKKKKKKKKKKKKKKKO!", &p[0], &p[1], &p[2], &p[3], &p[4], &p[5], &p[6], &p[7], &p[8], &p[9], &p[10], &p[11], &p[12],
                          &p[13], &p[14], &p[15], &p[16], &p[17], &PyType_Type, &axis)) return nullptr;
    attn_dense = (decltype(attn_dense))p[0];
    attn_block_sparse = (decltype(attn_block_sparse))p[1];
    attn_joint = (decltype(attn_joint))p[2];
    attn_joint_select = (decltype(attn_joint_select))p[3];
    mask_select = (decltype(mask_select))p[4];
    cache_store = (decltype(cache_store))p[5];
    cache_reuse = (decltype(cache_reuse))p[6];
    layer_linear = (decltype(layer_linear))p[7];
    layer_linear_bytes = (decltype(layer_linear_bytes))p[8];
    layer_modulate = (decltype(layer_modulate))p[9];
    layer_table = (decltype(layer_table))p[10];
    layer_qk = (decltype(layer_qk))p[11];
    layer_rope = (decltype(layer_rope))p[12];
    rows_quantize = (decltype(rows_quantize))p[13];
    rows_modulate = (decltype(rows_modulate))p[14];
    int8_linear = (decltype(int8_linear))p[15];
    int8_linear_bytes = (decltype(int8_linear_bytes))p[16];
    attn_packed = (decltype(attn_packed))p[17];
    Py_INCREF(axis);
    Py_XSETREF(axis_type, (PyObject*)axis);
    PyObject* c = PyImport_ImportModule("torch._C");
    if (!c) return nullptr;
    Py_XSETREF(current_stream, PyObject_GetAttrString(c, "_cuda_getCurrentRawStream"));
    Py_DECREF(c);
    if (!current_stream) return nullptr;
    Py_RETURN_NONE;
}

// A C++ exception of a tensor's accessor ends as an exception of Python's.
template <PyObject* (*F)(PyObject*, PyObject* const*, Py_ssize_t)>
PyObject* guarded(PyObject* self, PyObject* const* a, Py_ssize_t n)
{
    try {
        return F(self, a, n);
    } catch (const std::exception& e) {
        PyErr_SetString(PyExc_RuntimeError, e.what());
        return nullptr;
    }
}
#define NATIVE(f) {#f, (PyCFunction)(void (*)(void))guarded<f>, METH_FASTCALL, nullptr}
PyMethodDef methods[] = {{"bind", bind, METH_VARARGS, nullptr}, NATIVE(dense), NATIVE(block_sparse), NATIVE(select), NATIVE(joint),
                         NATIVE(joint_select), NATIVE(store), NATIVE(reuse), NATIVE(linear), NATIVE(modulate), NATIVE(table),
                         NATIVE(qk_norm_rope), NATIVE(rope), NATIVE(quantize), NATIVE(modulate8), NATIVE(linear8),
                         NATIVE(packed_attention), {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "native_call", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

// built_for: the torch and the Python whose headers this was compiled with (binding.py takes no other)
PyMODINIT_FUNC PyInit_native_call(void)
{
    PyObject* m = PyModule_Create(&module);
    if (m && PyModule_AddStringConstant(m, "built_for", BUILT_FOR) < 0) { Py_DECREF(m); return nullptr; }
    return m;
}
