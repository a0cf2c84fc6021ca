// Argument marshalling of the token-mixer calls, and of the gradients, for Python: checks the tensors, fills the
// descriptor and calls the C entry points of libjetvit.so.  Host time of a call, launches included,
// through ctypes structures / here: window or full attention 10.3 / 3.9 us, linear attention
// 13.7 / 7.4 us, the block with generated filters 25.4 / 20.3 us, where the kernels of a small problem take about 10.
// Only the ordinary forms are marshalled here: torch tensors with memory, pairs as tuples or lists.
// Every function returns the entry point's status, or None for arguments of any other form, valid
// or not, which binding.py then takes through ctypes: what is accepted, and the exceptions of what
// is not, are those of that path.  The interpreter lock is released around the entry points, as
// ctypes does, so that a launch that waits for room in the queue holds up no other thread.
#include <Python.h>

#include <ATen/hip/impl/HIPStreamMasqueradingAsCUDA.h>
#include <c10/hip/HIPFunctions.h>
#include <torch/csrc/autograd/python_variable.h>

#include "jetvit.h"

namespace {

// The readers below return false (or null) for a form that is left to binding.py; a Python error
// they leave set is cleared by `guarded`.
const at::Tensor *tensor_arg(PyObject *obj) { return THPVariable_Check(obj) ? &THPVariable_Unpack(obj) : nullptr; }

bool dtype_code(const at::Tensor &t, jv_dtype *out) {
    if (t.scalar_type() == at::kFloat) *out = JV_F32;
    else if (t.scalar_type() == at::kBFloat16) *out = JV_BF16;
    else return false;
    return true;
}

bool int_arg(PyObject *obj, int32_t *out) {
    const long x = PyLong_AsLong(obj);
    *out = (int32_t)x;
    return x == *out && !(x == -1 && PyErr_Occurred());
}

bool float_arg(PyObject *obj, float *out) {
    const double x = PyFloat_AsDouble(obj);
    *out = (float)x;
    return !(x == -1.0 && PyErr_Occurred());
}

// Items of a tuple or list of exactly n (borrowed references), or null.
PyObject **items_arg(PyObject *seq, Py_ssize_t n) {
    if (!PyTuple_Check(seq) && !PyList_Check(seq)) return nullptr;
    return PySequence_Fast_GET_SIZE(seq) == n ? PySequence_Fast_ITEMS(seq) : nullptr;
}

bool pair_arg(PyObject *seq, int32_t *a, int32_t *b) {
    PyObject **items = items_arg(seq, 2);
    return items && int_arg(items[0], a) && int_arg(items[1], b);
}

struct Call {
    jv_attn_desc desc;
    const void *q, *k, *v;
    void *o, *stream;
};

bool stream_arg(PyObject *obj, void **stream) {
    if (obj == Py_None) {
        *stream = at::hip::getCurrentHIPStreamMasqueradingAsCUDA().stream();
        return true;
    }
    PyObject *raw = PyObject_GetAttrString(obj, "cuda_stream");
    if (!raw) return false;
    *stream = PyLong_AsVoidPtr(raw);
    Py_DECREF(raw);
    return !PyErr_Occurred();
}

// args: q, k, v, o, grid
bool mixer_args(PyObject *const *args, PyObject *stream, Call *c) {
    const at::Tensor *t[4];
    for (int i = 0; i < 4; ++i)
        if (!(t[i] = tensor_arg(args[i]))) return false;
    jv_attn_desc &d = c->desc;
    if (!pair_arg(args[4], &d.grid_h, &d.grid_w) || t[0]->dim() != 4) return false;
    const auto shape = t[0]->sizes();
    const int64_t prefix = shape[2] - (int64_t)d.grid_h * d.grid_w;
    if (prefix < 0 || prefix != (int32_t)prefix) return false;
    jv_strides *strides[4] = {&d.q, &d.k, &d.v, &d.o};
    for (int i = 0; i < 4; ++i) {
        if (t[i]->sizes() != shape || !t[i]->is_cuda() || (i < 3 && t[i]->scalar_type() != t[0]->scalar_type())) return false;
        const auto s = t[i]->strides();
        if (s[3] != 1) return false;
        *strides[i] = {s[0], s[1], s[2]};
    }
    if (!dtype_code(*t[0], &d.dtype) || !dtype_code(*t[3], &d.o_dtype)) return false;
    for (int i : {0, 1, 3})
        if (shape[i] != (int32_t)shape[i]) return false;
    d.batch = (int32_t)shape[0];
    d.heads = (int32_t)shape[1];
    d.head_dim = (int32_t)shape[3];
    d.n_prefix = (int32_t)prefix;
    c->q = t[0]->data_ptr();
    c->k = t[1]->data_ptr();
    c->v = t[2]->data_ptr();
    c->o = t[3]->data_ptr();
    return stream_arg(stream, &c->stream);
}

// f() without the interpreter lock.
template <typename F>
PyObject *status_of(F f) {
    jv_status st;
    Py_BEGIN_ALLOW_THREADS
    st = f();
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(st);
}

bool workspace_arg(PyObject *obj, void **ptr, size_t *bytes) {
    const at::Tensor *t = tensor_arg(obj);
    if (!t) return false;
    *ptr = t->data_ptr();
    *bytes = t->nbytes();
    return true;
}

// (q, k, v, o, grid, eps, workspace, stream)
PyObject *linear_attn_fwd(PyObject *const *a) {
    Call c;
    float eps;
    void *ws;
    size_t bytes;
    if (!mixer_args(a, a[7], &c) || !float_arg(a[5], &eps) || !workspace_arg(a[6], &ws, &bytes)) return nullptr;
    return status_of([&] { return jv_linear_attn_fwd(&c.desc, c.q, c.k, c.v, c.o, eps, ws, bytes, c.stream); });
}

// One fp32 device tensor of the convolution's parameters; rows: the length of its first axis, if asked for.
bool param_arg(PyObject *obj, const float **out, int32_t *rows = nullptr) {
    const at::Tensor *t = tensor_arg(obj);
    if (!t || t->scalar_type() != at::kFloat || !t->is_cuda() || !t->is_contiguous()) return false;
    *out = (const float *)t->data_ptr();
    if (!rows) return true;
    if (t->dim() == 0 || t->size(0) != (int32_t)t->size(0)) return false;
    *rows = (int32_t)t->size(0);
    return true;
}

// static_kernel, squeeze, ksize, token as make_dwc_params of binding.py takes them
bool dwc_args(PyObject *kernel, PyObject *squeeze, PyObject *ksize, PyObject *token, jv_dwc_params *p) {
    *p = {JV_DWC_NONE, 3, 0, nullptr, nullptr, nullptr, nullptr, nullptr};
    if ((kernel != Py_None) + (squeeze != Py_None) + (token != Py_None) > 1 || !int_arg(ksize, &p->ksize)) return false;
    if (kernel != Py_None) {
        p->mode = JV_DWC_STATIC;
        return param_arg(kernel, &p->static_kernel);
    }
    PyObject *weights = squeeze != Py_None ? squeeze : token;
    if (weights == Py_None) return true;
    p->mode = squeeze != Py_None ? JV_DWC_SQUEEZE_DYNAMIC : JV_DWC_TOKEN_DYNAMIC;
    PyObject **w = items_arg(weights, 4);
    return w && param_arg(w[0], &p->w1, &p->hidden) && param_arg(w[1], &p->b1) && param_arg(w[2], &p->w2) && param_arg(w[3], &p->b2);
}

// (q, k, v, o, grid, eps, static_kernel, squeeze, ksize, token, focus_p, workspace, stream); focus_p 0: the ReLU map
PyObject *linear_block_fwd(PyObject *const *a) {
    Call c;
    jv_dwc_params dwc;
    float eps;
    int32_t focus;
    void *ws;
    size_t bytes;
    if (!mixer_args(a, a[12], &c) || !dwc_args(a[6], a[7], a[8], a[9], &dwc) || !float_arg(a[5], &eps) ||
        !int_arg(a[10], &focus) || !workspace_arg(a[11], &ws, &bytes))
        return nullptr;
    return status_of([&] {
        return focus == 0 ? jv_linear_block_fwd(&c.desc, c.q, c.k, c.v, c.o, eps, &dwc, ws, bytes, c.stream)
                          : jv_linear_block_focused_fwd(&c.desc, c.q, c.k, c.v, c.o, eps, focus, &dwc, ws, bytes, c.stream);
    });
}

// (q, k, v, o, grid, window, scale, stream)
PyObject *window_attn_fwd(PyObject *const *a) {
    Call c;
    int32_t wh, ww;
    float scale;
    if (!mixer_args(a, a[7], &c) || !pair_arg(a[5], &wh, &ww) || !float_arg(a[6], &scale)) return nullptr;
    return status_of([&] { return jv_window_attn_fwd(&c.desc, c.q, c.k, c.v, c.o, wh, ww, scale, c.stream); });
}

// (q, k, v, o, grid, scale, stream)
PyObject *full_attn_fwd(PyObject *const *a) {
    Call c;
    float scale;
    if (!mixer_args(a, a[6], &c) || !float_arg(a[5], &scale)) return nullptr;
    return status_of([&] { return jv_full_attn_fwd(&c.desc, c.q, c.k, c.v, c.o, scale, c.stream); });
}

// A tensor on the current device of `like`'s element type (like = null: any); None allowed where `absent` is given.
const at::Tensor *device_tensor(PyObject *obj, const at::Tensor *like, bool *absent = nullptr) {
    if (absent) {
        *absent = obj == Py_None;
        if (*absent) return nullptr;
    }
    const at::Tensor *t = tensor_arg(obj);
    return t && t->is_cuda() && t->get_device() == c10::hip::current_device() && (!like || t->scalar_type() == like->scalar_type()) ? t : nullptr;
}
bool bool_arg(PyObject *obj, bool *out) {
    const int x = PyObject_IsTrue(obj);
    *out = x > 0;
    return x >= 0;
}
// Memory of a number of bytes (a tensor without gaps), or None.
bool memory_arg(PyObject *obj, void **ptr, size_t *bytes) {
    bool absent;
    const at::Tensor *t = device_tensor(obj, nullptr, &absent);
    *ptr = t ? t->data_ptr() : nullptr;
    *bytes = t ? t->nbytes() : 0;
    return absent || (t && t->is_contiguous());
}
bool strided_arg(const at::Tensor *t, jv_strides *out, const at::Tensor *like = nullptr) {
    if (!t || t->dim() != 4 || t->stride(3) != 1 || (like && t->sizes() != like->sizes())) return false;
    *out = {t->stride(0), t->stride(1), t->stride(2)};
    return true;
}
bool lengths_arg(PyObject *obj, int64_t batch, const int32_t **out) {
    bool absent;
    const at::Tensor *t = device_tensor(obj, nullptr, &absent);
    *out = t ? (const int32_t *)t->data_ptr() : nullptr;
    return absent || (t && t->scalar_type() == at::kInt && t->dim() == 1 && t->size(0) == batch && t->is_contiguous());
}
// Four contiguous fp32 vectors of one shape.
bool vectors_arg(PyObject *obj, c10::IntArrayRef *shape, const float *(&out)[4], bool first) {
    PyObject **items = items_arg(obj, 4);
    if (!items) return false;
    for (int i = 0; i < 4; ++i) {
        const at::Tensor *t = device_tensor(items[i], nullptr);
        if (!t || t->scalar_type() != at::kFloat || !t->is_contiguous()) return false;
        if (first && i == 0) *shape = t->sizes();
        if (t->sizes() != *shape) return false;
        out[i] = (const float *)t->data_ptr();
    }
    return true;
}

struct DiffCall {
    jv_diff_attn_desc desc;
    jv_diff_lambda lambda;
    const at::Tensor *q, *k, *v, *o;
    c10::IntArrayRef shape;
    float scale;
    void *stream;
};
// args: q, k, v, lam, o; lambda_init, scale, causal, q_lengths, k_lengths; stream
bool diff_args(PyObject *const *a, PyObject *const *more, PyObject *stream, DiffCall *c) {
    c->desc = {};
    jv_diff_attn_desc &d = c->desc;
    bool causal;
    if (!(c->q = device_tensor(a[0], nullptr)) || !(c->k = device_tensor(a[1], c->q)) || !(c->v = device_tensor(a[2], c->q)) || !(c->o = device_tensor(a[4], nullptr)) ||
        !strided_arg(c->q, &d.q) || !strided_arg(c->k, &d.k) || !strided_arg(c->v, &d.v, c->k) || !strided_arg(c->o, &d.o, c->q) ||
        !dtype_code(*c->q, &d.dtype) || !dtype_code(*c->o, &d.o_dtype) || !float_arg(more[0], &c->lambda.init) || !float_arg(more[1], &c->scale) ||
        !bool_arg(more[2], &causal) || !lengths_arg(more[3], c->q->size(0), &d.q_lengths) || !lengths_arg(more[4], c->q->size(0), &d.k_lengths))
        return false;
    const auto q = c->q->sizes(), k = c->k->sizes();
    if (k[0] != q[0] || k[3] != q[3]) return false;
    for (int64_t x : {q[0], q[1], q[2], q[3], k[1], k[2]})
        if (x != (int32_t)x) return false;
    d.batch = (int32_t)q[0];
    d.heads = (int32_t)q[1];
    d.kv_heads = (int32_t)k[1];
    d.n_q = (int32_t)q[2];
    d.n_k = (int32_t)k[2];
    d.head_dim = (int32_t)q[3];
    d.causal = causal;
    const float *vec[4];
    if (!vectors_arg(a[3], &c->shape, vec, true)) return false;
    const int64_t half = q[3] / 2;
    if (!(c->shape == c10::IntArrayRef({half}) || c->shape == c10::IntArrayRef({q[1], half}))) return false;
    c->lambda.q1 = vec[0];
    c->lambda.k1 = vec[1];
    c->lambda.q2 = vec[2];
    c->lambda.k2 = vec[3];
    c->lambda.per_head = c->shape.size() == 2;
    return stream_arg(stream, &c->stream);
}

// (q, k, v, lam, o, lambda_init, scale, causal, q_lengths, k_lengths, saved, workspace, stream)
PyObject *diff_attn_fwd(PyObject *const *a) {
    DiffCall c;
    void *saved, *ws;
    size_t saved_bytes, bytes;
    if (!diff_args(a, a + 5, a[12], &c) || !memory_arg(a[10], &saved, &saved_bytes) || !memory_arg(a[11], &ws, &bytes)) return nullptr;
    return status_of([&] {
        return jv_diff_attn_fwd(&c.desc, c.q->data_ptr(), c.k->data_ptr(), c.v->data_ptr(), &c.lambda, c.o->data_ptr(), c.scale, saved, saved_bytes, ws, bytes, c.stream);
    });
}

// (q, k, v, lam, o, saved, d_o, d_q, d_k, d_v, d_lam, lambda_init, scale, causal, q_lengths, k_lengths, workspace, stream)
PyObject *diff_attn_bwd(PyObject *const *a) {
    DiffCall c;
    jv_diff_attn_grads g = {};
    void *saved, *ws;
    size_t saved_bytes, bytes;
    if (!diff_args(a, a + 11, a[17], &c) || !memory_arg(a[5], &saved, &saved_bytes) || !memory_arg(a[16], &ws, &bytes)) return nullptr;
    const at::Tensor *d_o = device_tensor(a[6], c.q), *d_q = device_tensor(a[7], c.q), *d_k = device_tensor(a[8], c.q), *d_v = device_tensor(a[9], c.q);
    if (!strided_arg(d_o, &g.d_o_strides, c.q) || !strided_arg(d_q, &g.d_q_strides, c.q) || !strided_arg(d_k, &g.d_k_strides, c.k) || !strided_arg(d_v, &g.d_v_strides, c.v))
        return nullptr;
    g.d_o = d_o->data_ptr();
    g.d_q = d_q->data_ptr();
    g.d_k = d_k->data_ptr();
    g.d_v = d_v->data_ptr();
    if (a[10] != Py_None) {
        const float *vec[4];
        if (!vectors_arg(a[10], &c.shape, vec, false)) return nullptr;
        g.d_q1 = (float *)vec[0];
        g.d_k1 = (float *)vec[1];
        g.d_q2 = (float *)vec[2];
        g.d_k2 = (float *)vec[3];
    }
    return status_of([&] {
        return jv_diff_attn_bwd(&c.desc, c.q->data_ptr(), c.k->data_ptr(), c.v->data_ptr(), &c.lambda, c.o->data_ptr(), saved, saved_bytes, &g, c.scale, ws, bytes, c.stream);
    });
}

// (x, gamma, dy, dx, dgamma, dbeta, eps, residual, workspace, stream)
PyObject *layernorm_bwd(PyObject *const *a) {
    bool no_dgamma, no_dbeta, no_residual;
    const at::Tensor *x = device_tensor(a[0], nullptr), *gamma = device_tensor(a[1], nullptr), *dy = device_tensor(a[2], nullptr);
    if (!x || !gamma || !dy) return nullptr;
    const at::Tensor *dx = device_tensor(a[3], x), *dgamma = device_tensor(a[4], gamma, &no_dgamma), *dbeta = device_tensor(a[5], gamma, &no_dbeta);
    const at::Tensor *residual = device_tensor(a[7], x, &no_residual);
    if (!dx || !(dgamma || no_dgamma) || !(dbeta || no_dbeta) || !(residual || no_residual) || x->dim() != 2 || gamma->scalar_type() != at::kFloat) return nullptr;
    for (const at::Tensor *t : {x, dy, dx, residual})
        if (t && (!t->is_contiguous() || t->sizes() != x->sizes())) return nullptr;
    const int64_t rows = x->size(0), cols = x->size(1);
    for (const at::Tensor *t : {gamma, dgamma, dbeta})
        if (t && (!t->is_contiguous() || t->sizes() != c10::IntArrayRef({cols}))) return nullptr;
    jv_dtype x_type, dy_type;
    float eps;
    void *ws, *stream;
    size_t bytes;
    if (cols != (int32_t)cols || !dtype_code(*x, &x_type) || !dtype_code(*dy, &dy_type) || !float_arg(a[6], &eps) || !memory_arg(a[8], &ws, &bytes) || !stream_arg(a[9], &stream))
        return nullptr;
    auto ptr = [](const at::Tensor *t) { return t ? t->data_ptr() : nullptr; };
    return status_of([&] {
        return jv_layernorm_bwd(x->data_ptr(), (const float *)gamma->data_ptr(), dy->data_ptr(), ptr(residual), dx->data_ptr(), (float *)ptr(dgamma), (float *)ptr(dbeta), rows,
                                (int32_t)cols, eps, x_type, dy_type, ws, bytes, stream);
    });
}

// Tensors without memory of their own (under tracing or vmap) throw where their pointer or strides
// are asked for, and torch where it has no device for the current stream: left to binding.py too.
// Nothing throws behind an entry point, so no call is made twice.
template <PyObject *(*F)(PyObject *const *), Py_ssize_t ARGS>
PyObject *guarded(PyObject *, PyObject *const *a, Py_ssize_t n) {
    if (n != ARGS) {
        PyErr_SetString(PyExc_TypeError, "wrong number of arguments");
        return nullptr;
    }
    try {
        if (PyObject *status = F(a)) return status;
    } catch (const std::exception &) {
    }
    PyErr_Clear();
    Py_RETURN_NONE;
}

PyMethodDef methods[] = {
    {"linear_attn_fwd", (PyCFunction)(void *)guarded<linear_attn_fwd, 8>, METH_FASTCALL, nullptr},
    {"linear_block_fwd", (PyCFunction)(void *)guarded<linear_block_fwd, 13>, METH_FASTCALL, nullptr},
    {"window_attn_fwd", (PyCFunction)(void *)guarded<window_attn_fwd, 8>, METH_FASTCALL, nullptr},
    {"full_attn_fwd", (PyCFunction)(void *)guarded<full_attn_fwd, 7>, METH_FASTCALL, nullptr},
    {"diff_attn_fwd", (PyCFunction)(void *)guarded<diff_attn_fwd, 13>, METH_FASTCALL, nullptr},
    {"diff_attn_bwd", (PyCFunction)(void *)guarded<diff_attn_bwd, 18>, METH_FASTCALL, nullptr},
    {"layernorm_bwd", (PyCFunction)(void *)guarded<layernorm_bwd, 10>, METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr},
};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_native", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__native(void) { return PyModule_Create(&module); }
