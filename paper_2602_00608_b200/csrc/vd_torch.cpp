// The transformer-block operators' way from torch tensors to the C entry points (vd_block.h) without Python in between: types,
// sizes, strides and addresses are read from the tensors and handed over.  A token's operators run for four microseconds;
// reading ten tensors' attributes from Python takes as long.  Whatever is not plainly right here is left to the Python path
// (the functions return None), which says what is wrong with it.  Nothing is kept between calls.
#include <Python.h>
#include <c10/cuda/CUDAFunctions.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include <cmath>

#include "vd_block.h"

namespace {

decltype(&vd_op_cross_attention) xattn_fn = nullptr;
decltype(&vd_op_rotary) rotary_fn = nullptr;
decltype(&vd_op_gate_norm) norm_fn = nullptr;

constexpr int64_t INT_LIMIT = int64_t(1) << 31;

// a tensor argument: null for None, `ok` false for anything else that is no tensor
struct Arg {
    const at::Tensor* t = nullptr;
    bool ok = true;
    explicit Arg(PyObject* o) {
        if (o == Py_None) return;
        ok = THPVariable_Check(o);
        if (ok) t = &THPVariable_Unpack(o);
    }
    void* ptr() const { return t ? t->data_ptr() : nullptr; }
};

int dtype_of(const at::Tensor& t) {
    const auto s = t.scalar_type();
    return s == at::kBFloat16 ? VD_BF16 : s == at::kFloat ? VD_F32 : -1;
}
// on this device (which is the current one), sizes within int32
bool here(const at::Tensor& t, c10::DeviceIndex device) {
    if (!t.is_cuda() || t.get_device() != device) return false;
    for (const auto n : t.sizes())
        if (n >= INT_LIMIT) return false;
    return true;
}
bool is_text(PyObject* o, const char* text) { return PyUnicode_Check(o) && PyUnicode_CompareWithASCIIString(o, text) == 0; }

PyObject* finish(int status) { return PyLong_FromLong(status); }
#define LEAVE_UNLESS(c) do { if (!(c)) { PyErr_Clear(); Py_RETURN_NONE; } } while (0)

PyObject* bind(PyObject*, PyObject* const* a, Py_ssize_t n) {
    if (n != 3) { PyErr_SetString(PyExc_TypeError, "three addresses"); return nullptr; }
    xattn_fn = (decltype(xattn_fn))PyLong_AsVoidPtr(a[0]);
    rotary_fn = (decltype(rotary_fn))PyLong_AsVoidPtr(a[1]);
    norm_fn = (decltype(norm_fn))PyLong_AsVoidPtr(a[2]);
    if (PyErr_Occurred()) return nullptr;
    Py_RETURN_NONE;
}

// q, k, v, kv_lens, scale, out, impl
PyObject* cross_attention(PyObject*, PyObject* const* a, Py_ssize_t n) {
    LEAVE_UNLESS(n == 7 && xattn_fn);
    const Arg q(a[0]), k(a[1]), v(a[2]), lens(a[3]), o(a[5]);
    LEAVE_UNLESS(q.ok && k.ok && v.ok && lens.ok && o.ok && q.t && k.t && v.t && o.t);
    const auto device = c10::cuda::current_device();
    for (const Arg* x : {&q, &k, &v, &o}) LEAVE_UNLESS(x->t->dim() == 4 && here(*x->t, device) && dtype_of(*x->t) >= 0 && dtype_of(*x->t) == dtype_of(*q.t));
    const auto qs = q.t->sizes(), ks = k.t->sizes(), sq = q.t->strides(), sk = k.t->strides(), sv = v.t->strides(), so = o.t->strides();
    LEAVE_UNLESS(ks == v.t->sizes() && qs == o.t->sizes() && ks[0] == qs[0] && ks[3] == qs[3]);
    LEAVE_UNLESS(qs[3] <= 1 || (sq[3] == 1 && sk[3] == 1 && sv[3] == 1 && so[3] == 1));
    LEAVE_UNLESS(!lens.t || (here(*lens.t, device) && lens.t->scalar_type() == at::kInt && lens.t->dim() == 1 && lens.t->size(0) == qs[0] && lens.t->is_contiguous()));
    vd_xattn_desc d = {};
    d.struct_size = sizeof(d);
    d.dtype = dtype_of(*q.t);
    d.batch = (int32_t)qs[0]; d.q_len = (int32_t)qs[1]; d.kv_len = (int32_t)ks[1];
    d.heads = (int32_t)qs[2]; d.kv_heads = (int32_t)ks[2]; d.head_dim = (int32_t)qs[3];
    LEAVE_UNLESS(PyLong_Check(a[6]));
    const long impl = PyLong_AsLong(a[6]);
    LEAVE_UNLESS(!PyErr_Occurred() && impl >= 0 && impl < 16);
    d.impl = (int32_t)impl;
    LEAVE_UNLESS(a[4] == Py_None ? d.head_dim > 0 : PyFloat_Check(a[4]));
    d.scale = (float)(a[4] == Py_None ? std::pow((double)d.head_dim, -0.5) : PyFloat_AS_DOUBLE(a[4]));
    d.q_batch = sq[0]; d.q_token = sq[1]; d.q_head = sq[2];
    d.k_batch = sk[0]; d.k_token = sk[1]; d.k_head = sk[2];
    d.v_batch = sv[0]; d.v_token = sv[1]; d.v_head = sv[2];
    d.o_batch = so[0]; d.o_token = so[1]; d.o_head = so[2];
    return finish(xattn_fn(&d, q.ptr(), k.ptr(), v.ptr(), (const int32_t*)lens.ptr(), o.ptr(), c10::cuda::getCurrentCUDAStream(device).stream()));
}

// x, freqs, positions, layout, axis_pairs (tuple or None), amplitude, first_position, out
PyObject* rotary(PyObject*, PyObject* const* a, Py_ssize_t n) {
    LEAVE_UNLESS(n == 8 && rotary_fn);
    const Arg x(a[0]), f(a[1]), pos(a[2]), y(a[7]);
    LEAVE_UNLESS(x.ok && f.ok && pos.ok && y.ok && x.t && f.t && y.t);
    const auto device = c10::cuda::current_device();
    LEAVE_UNLESS(x.t->dim() == 4 && here(*x.t, device) && here(*y.t, device) && here(*f.t, device));
    LEAVE_UNLESS(dtype_of(*x.t) >= 0 && x.t->scalar_type() == y.t->scalar_type() && x.t->sizes() == y.t->sizes());
    LEAVE_UNLESS(f.t->scalar_type() == at::kDouble && f.t->dim() == 1 && f.t->is_contiguous() && f.t->size(0) <= 512);
    vd_rotary_desc d = {};
    d.struct_size = sizeof(d);
    d.axes = 1;
    d.axis_pairs[0] = (int32_t)f.t->size(0);
    if (a[4] != Py_None) {
        LEAVE_UNLESS(PyTuple_Check(a[4]) && PyTuple_GET_SIZE(a[4]) >= 1 && PyTuple_GET_SIZE(a[4]) <= VD_ROTARY_MAX_AXES);
        d.axes = (int32_t)PyTuple_GET_SIZE(a[4]);
        for (int i = 0; i < d.axes; ++i) {
            PyObject* p = PyTuple_GET_ITEM(a[4], i);
            LEAVE_UNLESS(PyLong_Check(p));
            const long v = PyLong_AsLong(p);
            LEAVE_UNLESS(!PyErr_Occurred() && v >= 0 && v <= 512);
            d.axis_pairs[i] = (int32_t)v;
        }
    }
    const auto s = x.t->sizes(), sx = x.t->strides(), sy = y.t->strides();
    LEAVE_UNLESS(s[3] <= 1 || (sx[3] == 1 && sy[3] == 1));
    d.dtype = dtype_of(*x.t);
    d.batch = (int32_t)s[0]; d.tokens = (int32_t)s[1]; d.heads = (int32_t)s[2]; d.head_dim = (int32_t)s[3];
    d.rotary_dim = (int32_t)(2 * f.t->size(0));
    LEAVE_UNLESS(is_text(a[3], "half") || is_text(a[3], "interleaved"));
    d.layout = is_text(a[3], "half") ? VD_ROTARY_HALF : VD_ROTARY_INTERLEAVED;
    LEAVE_UNLESS(PyFloat_Check(a[5]) && PyLong_Check(a[6]));
    d.amplitude = (float)PyFloat_AS_DOUBLE(a[5]);
    d.first_position = PyLong_AsLongLong(a[6]);
    LEAVE_UNLESS(!PyErr_Occurred());
    if (pos.t) {
        const auto ps = pos.t->sizes();
        LEAVE_UNLESS(here(*pos.t, device) && pos.t->scalar_type() == at::kInt && (ps.size() == 3 || (ps.size() == 2 && d.axes == 1)) && ps[0] == s[0] && ps[1] == s[1]);
        LEAVE_UNLESS(ps.size() == 2 || (ps[2] == d.axes && (d.axes == 1 || pos.t->stride(2) == 1)));
        d.pos_batch = pos.t->stride(0);
        d.pos_token = pos.t->stride(1);
    }
    d.x_batch = sx[0]; d.x_token = sx[1]; d.x_head = sx[2];
    d.y_batch = sy[0]; d.y_token = sy[1]; d.y_head = sy[2];
    return finish(rotary_fn(&d, x.ptr(), (const int32_t*)pos.ptr(), (const double*)f.ptr(), y.ptr(), c10::cuda::getCurrentCUDAStream(device).stream()));
}

// x, h, gate, scale, shift, kind, eps, weight, bias, post_norm, post_weight, residual_scale, mod_tokens (int or None), x_out, y
PyObject* gate_norm(PyObject*, PyObject* const* a, Py_ssize_t n) {
    LEAVE_UNLESS(n == 15 && norm_fn);
    const Arg x(a[0]), h(a[1]), gate(a[2]), scale(a[3]), shift(a[4]), weight(a[7]), bias(a[8]), post(a[10]), xo(a[13]), y(a[14]);
    for (const Arg* t : {&x, &h, &gate, &scale, &shift, &weight, &bias, &post, &xo, &y}) LEAVE_UNLESS(t->ok);
    LEAVE_UNLESS(x.t && x.t->dim() == 3);
    const auto device = c10::cuda::current_device();
    const auto s = x.t->sizes();
    vd_gate_norm_desc d = {};
    d.struct_size = sizeof(d);
    d.batch = (int32_t)s[0]; d.tokens = (int32_t)s[1]; d.channels = (int32_t)s[2];
    int64_t mod_tokens = s[1] > 0 ? s[1] : 1;
    if (a[12] != Py_None) {
        LEAVE_UNLESS(PyLong_Check(a[12]));
        mod_tokens = PyLong_AsLongLong(a[12]);
        LEAVE_UNLESS(!PyErr_Occurred() && mod_tokens >= 1 && mod_tokens < INT_LIMIT);
    }
    d.mod_tokens = (int32_t)mod_tokens;
    struct Row { const Arg* t; int64_t *batch, *token; };
    for (const Row& r : {Row{&x, &d.x_batch, &d.x_token}, Row{&h, &d.h_batch, &d.h_token}, Row{&xo, &d.xo_batch, &d.xo_token}, Row{&y, &d.y_batch, &d.y_token}}) {
        if (!r.t->t) continue;
        const at::Tensor& t = *r.t->t;
        LEAVE_UNLESS(here(t, device) && t.sizes() == s && dtype_of(t) >= 0 && (s[2] <= 1 || t.stride(2) == 1));
        *r.batch = t.stride(0);
        *r.token = t.stride(1);
    }
    LEAVE_UNLESS(!xo.t || xo.t->scalar_type() == x.t->scalar_type());
    d.x_dtype = dtype_of(*x.t);
    d.h_dtype = h.t ? dtype_of(*h.t) : d.x_dtype;
    d.y_dtype = y.t ? dtype_of(*y.t) : d.x_dtype;
    d.mod_dtype = VD_F32;
    const int64_t groups = (s[1] + mod_tokens - 1) / mod_tokens;
    int mod = -1;
    for (const Row& r : {Row{&gate, &d.gate_batch, &d.gate_group}, Row{&scale, &d.scale_batch, &d.scale_group}, Row{&shift, &d.shift_batch, &d.shift_group}}) {
        if (!r.t->t) continue;
        const at::Tensor& t = *r.t->t;
        LEAVE_UNLESS(here(t, device) && t.dim() == 3 && t.size(0) == s[0] && t.size(1) == groups && t.size(2) == s[2] && (s[2] <= 1 || t.stride(2) == 1));
        LEAVE_UNLESS(dtype_of(t) >= 0 && (mod < 0 || mod == dtype_of(t)));
        d.mod_dtype = mod = dtype_of(t);
        *r.batch = t.stride(0);
        *r.token = t.stride(1);
    }
    for (const Arg* w : {&weight, &bias, &post})
        LEAVE_UNLESS(!w->t || (here(*w->t, device) && w->t->scalar_type() == at::kFloat && w->t->dim() == 1 && w->t->size(0) == s[2] && w->t->is_contiguous()));
    LEAVE_UNLESS(is_text(a[5], "layer") || is_text(a[5], "rms"));
    d.norm = is_text(a[5], "layer") ? VD_NORM_LAYER : VD_NORM_RMS;
    LEAVE_UNLESS(PyFloat_Check(a[6]) && PyBool_Check(a[9]) && PyFloat_Check(a[11]));
    d.eps = (float)PyFloat_AS_DOUBLE(a[6]);
    d.post_norm = a[9] == Py_True;
    d.residual_scale = (float)PyFloat_AS_DOUBLE(a[11]);
    return finish(norm_fn(&d, x.ptr(), h.ptr(), (const float*)post.ptr(), gate.ptr(), xo.ptr(), (const float*)weight.ptr(), (const float*)bias.ptr(), scale.ptr(),
                          shift.ptr(), y.ptr(), c10::cuda::getCurrentCUDAStream(device).stream()));
}

// C++ exceptions of the tensor library end here: the Python path meets what raised them
template <PyObject* (*F)(PyObject*, PyObject* const*, Py_ssize_t)> PyObject* guarded(PyObject* self, PyObject* const* a, Py_ssize_t n) {
    try {
        return F(self, a, n);
    } catch (...) {
        PyErr_Clear();
        Py_RETURN_NONE;
    }
}

PyMethodDef methods[] = {
    {"bind", (PyCFunction)(void (*)(void))guarded<bind>, METH_FASTCALL, "addresses of vd_op_cross_attention, vd_op_rotary, vd_op_gate_norm"},
    {"cross_attention", (PyCFunction)(void (*)(void))guarded<cross_attention>, METH_FASTCALL, "status, or None: not plainly right"},
    {"rotary", (PyCFunction)(void (*)(void))guarded<rotary>, METH_FASTCALL, "status, or None: not plainly right"},
    {"gate_norm", (PyCFunction)(void (*)(void))guarded<gate_norm>, METH_FASTCALL, "status, or None: not plainly right"},
    {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_vd_torch", "torch tensors to libvd's block operators", -1, methods};

}  // namespace

PyMODINIT_FUNC PyInit__vd_torch() { return PyModule_Create(&module); }
