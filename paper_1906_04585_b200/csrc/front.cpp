// The short way from torch tensors to the sequence-policy operators, as a CPython module.
//
// A call on small tensors (one acting step) is bound by the host: a launch takes some 3 us, the checks and the argument
// struct in Python twice that and more.  These functions do the same for tensors that are as they should be, and return
// None for anything else - a wrong type or shape, a stride that needs thought, a refusal by the library - which the Python
// code then says in words (refused calls enqueue nothing, so asking twice is safe).  No operator's work is done here.
#include <Python.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include <ATen/ops/empty.h>
#include <c10/cuda/CUDAFunctions.h>
#include <c10/cuda/CUDAStream.h>

#include "gala.h"

namespace {

using at::Tensor;

// -1: not an element type of the operators
int type_of(const Tensor& t) {
    switch (t.scalar_type()) {
        case at::kFloat: return GALA_F32;
        case at::kBFloat16: return GALA_BF16;
        case at::kHalf: return GALA_F16;
        default: return -1;
    }
}

// a size that the library takes as an int
bool fits(int64_t n) { return n <= INT32_MAX; }

// Arguments of one call.  `good` turns false at the first one that is not simple.
struct Call {
    const Tensor& like;
    int dev;
    bool good = true;
    explicit Call(const Tensor& x) : like(x), dev(x.is_cuda() ? x.get_device() : -1) { good = dev >= 0 && dev == c10::cuda::current_device(); }

    const Tensor* tensor(PyObject* o, at::ScalarType type) {      // nullptr: None, or not simple
        if (o == Py_None) return nullptr;
        if (!THPVariable_Check(o)) {
            good = false;
            return nullptr;
        }
        const Tensor& t = THPVariable_Unpack(o);
        if (!t.is_cuda() || t.get_device() != dev || t.scalar_type() != type) good = false;
        return good ? &t : nullptr;
    }
    // a matrix of this shape with contiguous columns
    void* rows(const Tensor& t, int64_t n, int64_t m, long long& ld) {
        if (t.dim() != 2 || t.size(0) != n || t.size(1) != m || (m > 1 && t.stride(1) != 1)) {
            good = false;
            return nullptr;
        }
        ld = n > 1 ? t.stride(0) : (m + 7) / 8 * 8;      // a single row may carry any stride
        return t.data_ptr();
    }
    void* rows(PyObject* o, int64_t n, int64_t m, long long& ld) {
        const Tensor* t = tensor(o, like.scalar_type());
        return t ? rows(*t, n, m, ld) : nullptr;
    }
    // a contiguous tensor of this many dimensions and this shape
    void* flat(const Tensor& t, int64_t n, int64_t m = -1) {
        if (t.dim() != (m < 0 ? 1 : 2) || t.size(0) != n || (m >= 0 && t.size(1) != m) || !t.is_contiguous()) {
            good = false;
            return nullptr;
        }
        return t.data_ptr();
    }
    void* flat(PyObject* o, at::ScalarType type, int64_t n, int64_t m = -1) {
        const Tensor* t = tensor(o, type);
        return t ? flat(*t, n, m) : nullptr;
    }
    // [steps][batch][dim] with contiguous channels
    void* steps(const Tensor& t, int64_t T, int64_t N, int64_t D, long long& st, long long& sb) {
        if (t.dim() != 3 || t.size(0) != T || t.size(1) != N || t.size(2) != D || (D > 1 && t.stride(2) != 1)) {
            good = false;
            return nullptr;
        }
        st = t.stride(0);
        sb = t.stride(1);
        return t.data_ptr();
    }
    Tensor make(at::IntArrayRef shape, at::ScalarType type) const { return at::empty(shape, at::TensorOptions().dtype(type).device(like.device())); }
    void* stream() const { return c10::cuda::getCurrentCUDAStream(dev).stream(); }
};

PyObject* keep(PyObject* o) {
    Py_INCREF(o);
    return o;
}
PyObject* wrap_or(PyObject* given, const Tensor& made) { return given != Py_None ? keep(given) : THPVariable_Wrap(made); }
PyObject* four(PyObject* a, PyObject* b, PyObject* c, PyObject* d) {
    PyObject* t = PyTuple_New(4);
    PyTuple_SET_ITEM(t, 0, a);
    PyTuple_SET_ITEM(t, 1, b);
    PyTuple_SET_ITEM(t, 2, c);
    PyTuple_SET_ITEM(t, 3, d);
    return t;
}

// What torch throws leaves as torch's own Python errors (out of memory among them).
#define BEGIN try {
#define END                                                                     \
    }                                                                           \
    catch (...) {                                                               \
        torch::translate_exception_to_python(std::current_exception());         \
        return nullptr;                                                         \
    }

// layer_norm(x, weight, bias, eps, residual, out, sum_out)
PyObject* layer_norm(PyObject*, PyObject* const* a, Py_ssize_t n) {
    BEGIN
    if (n != 7 || !THPVariable_Check(a[0])) Py_RETURN_NONE;
    const Tensor& x = THPVariable_Unpack(a[0]);
    Call c(x);
    gala_layer_norm_args g = {};
    g.dtype = type_of(x);
    if (!c.good || g.dtype < 0 || x.dim() != 2) Py_RETURN_NONE;
    const int64_t R = x.size(0), C = x.size(1);
    if (!fits(C)) Py_RETURN_NONE;
    at::ScalarType wt = x.scalar_type();
    for (int i = 2; i > 0; i--)
        if (THPVariable_Check(a[i])) wt = THPVariable_Unpack(a[i]).scalar_type();
    g.wdtype = wt == at::kFloat ? (int)GALA_F32 : wt == x.scalar_type() ? g.dtype : -1;
    g.rows = R;
    g.cols = (int)C;
    g.eps = (float)PyFloat_AsDouble(a[3]);
    if (PyErr_Occurred()) return nullptr;
    g.x = c.rows(x, R, C, g.x_ld);
    g.weight = c.flat(a[1], wt, C);
    g.bias = c.flat(a[2], wt, C);
    Tensor y, s;
    if (a[5] == Py_None) {
        y = c.make({R, C}, x.scalar_type());
        g.y = c.rows(y, R, C, g.y_ld);
    } else {
        g.y = c.rows(a[5], R, C, g.y_ld);
    }
    const bool residual = a[4] != Py_None;
    if (residual) {
        g.residual = c.rows(a[4], R, C, g.residual_ld);
        if (a[6] == Py_None) {
            s = c.make({R, C}, x.scalar_type());
            g.sum = c.rows(s, R, C, g.sum_ld);
        } else {
            g.sum = c.rows(a[6], R, C, g.sum_ld);
        }
    } else if (a[6] != Py_None) {
        Py_RETURN_NONE;
    }
    if (!c.good) Py_RETURN_NONE;
    const Tensor stats = c.make({2, R}, at::kFloat);
    g.mean = stats.data_ptr<float>();
    g.rstd = g.mean + R;
    if (gala_layer_norm_forward(&g, c.stream(), nullptr, 0) < 0) Py_RETURN_NONE;
    return four(wrap_or(a[5], y), residual ? wrap_or(a[6], s) : keep(a[0]), THPVariable_Wrap(stats.select(0, 0)), THPVariable_Wrap(stats.select(0, 1)));
    END
}

// gated_recurrence(f, x, h0, done, out, h_last, status): without stored states
PyObject* gated_recurrence(PyObject*, PyObject* const* a, Py_ssize_t n) {
    BEGIN
    if (n != 7 || !THPVariable_Check(a[0]) || !THPVariable_Check(a[1])) Py_RETURN_NONE;
    const Tensor& x = THPVariable_Unpack(a[1]);
    Call c(x);
    gala_recurrence_args g = {};
    g.dtype = type_of(x);
    if (!c.good || g.dtype < 0 || x.dim() != 3) Py_RETURN_NONE;
    const int64_t T = x.size(0), N = x.size(1), D = x.size(2);
    g.steps = T;
    g.batch = N;
    g.dim = D;
    g.x = c.steps(x, T, N, D, g.x_t, g.x_b);
    const Tensor* f = c.tensor(a[0], x.scalar_type());
    if (!f) Py_RETURN_NONE;
    g.f = c.steps(*f, T, N, D, g.f_t, g.f_b);
    g.h0 = static_cast<const float*>(c.flat(a[2], at::kFloat, N, D));
    if (a[3] != Py_None) {
        if (!THPVariable_Check(a[3])) Py_RETURN_NONE;
        const at::ScalarType dt = THPVariable_Unpack(a[3]).scalar_type();
        if (dt != at::kByte && dt != at::kBool) Py_RETURN_NONE;
        const Tensor* d = c.tensor(a[3], dt);
        if (!d || d->dim() != 2 || d->size(0) != T || d->size(1) != N) Py_RETURN_NONE;
        g.done = static_cast<const unsigned char*>(d->data_ptr());
        g.done_t = d->stride(0);
        g.done_b = d->stride(1);
    }
    Tensor h, last;
    if (a[4] == Py_None) {
        h = c.make({T, N, D}, x.scalar_type());
        g.h = c.steps(h, T, N, D, g.h_t, g.h_b);
    } else {
        const Tensor* t = c.tensor(a[4], x.scalar_type());
        if (!t) Py_RETURN_NONE;
        g.h = c.steps(*t, T, N, D, g.h_t, g.h_b);
    }
    if (a[5] == Py_None) {
        last = c.make({N, D}, at::kFloat);
        g.h_last = last.data_ptr<float>();
    } else {
        g.h_last = static_cast<float*>(c.flat(a[5], at::kFloat, N, D));
    }
    g.status = static_cast<int*>(PyLong_AsVoidPtr(a[6]));
    if (PyErr_Occurred()) return nullptr;
    if (!c.good || gala_gated_recurrence_forward(&g, c.stream(), nullptr, 0) < 0) Py_RETURN_NONE;
    PyObject* t = PyTuple_New(3);
    PyTuple_SET_ITEM(t, 0, wrap_or(a[4], h));
    PyTuple_SET_ITEM(t, 1, wrap_or(a[5], last));
    PyTuple_SET_ITEM(t, 2, keep(Py_None));
    return t;
    END
}

// gated_ffn(x, w_gate, w_up, w_down, act, out, status): without stored projections
PyObject* gated_ffn(PyObject*, PyObject* const* a, Py_ssize_t n) {
    BEGIN
    if (n != 7 || !THPVariable_Check(a[0]) || !THPVariable_Check(a[1])) Py_RETURN_NONE;
    const Tensor& x = THPVariable_Unpack(a[0]);
    Call c(x);
    gala_ffn_args g = {};
    g.dtype = type_of(x);
    if (!c.good || g.dtype < 0 || x.dim() != 2) Py_RETURN_NONE;
    const Tensor* wg = c.tensor(a[1], x.scalar_type());
    if (!wg || wg->dim() != 2) Py_RETURN_NONE;
    const int64_t R = x.size(0), D = x.size(1), F = wg->size(0);
    if (!fits(D) || !fits(F)) Py_RETURN_NONE;
    g.act = (int)PyLong_AsLong(a[4]);
    g.status = static_cast<int*>(PyLong_AsVoidPtr(a[6]));
    if (PyErr_Occurred()) return nullptr;
    g.rows = R;
    g.dim = (int)D;
    g.hidden = (int)F;
    g.x = c.rows(x, R, D, g.x_ld);
    g.w_gate = c.rows(*wg, F, D, g.w_gate_ld);
    g.w_up = c.rows(a[2], F, D, g.w_up_ld);
    g.w_down = c.rows(a[3], D, F, g.w_down_ld);
    Tensor y;
    if (a[5] == Py_None) {
        y = c.make({R, (D + 7) / 8 * 8}, x.scalar_type()).narrow(1, 0, D);
        g.y = c.rows(y, R, D, g.y_ld);
    } else {
        g.y = c.rows(a[5], R, D, g.y_ld);
    }
    if (!c.good || !g.w_up || !g.w_down) Py_RETURN_NONE;
    g.hidden_ld = (F + 7) / 8 * 8;
    const Tensor product = c.make({R, g.hidden_ld}, x.scalar_type());
    g.product = product.data_ptr();
    if (gala_gated_ffn_forward(&g, c.stream(), nullptr, 0) < 0) Py_RETURN_NONE;
    return wrap_or(a[5], y);
    END
}

// sample(logits, uniforms, temperature, top_k, top_p, min_p, out, logprobs)
PyObject* sample(PyObject*, PyObject* const* a, Py_ssize_t n) {
    BEGIN
    if (n != 8 || !THPVariable_Check(a[0]) || a[1] == Py_None) Py_RETURN_NONE;
    const Tensor& l = THPVariable_Unpack(a[0]);
    Call c(l);
    gala_sample_args g = {};
    g.dtype = type_of(l);
    if (!c.good || g.dtype < 0 || l.dim() != 2) Py_RETURN_NONE;
    const int64_t R = l.size(0), V = l.size(1);
    if (!fits(V)) Py_RETURN_NONE;
    g.rows = R;
    g.vocab = (int)V;
    g.logits = c.rows(l, R, V, g.logits_ld);
    g.uniforms = static_cast<const float*>(c.flat(a[1], at::kFloat, R));
    g.temperature = static_cast<const float*>(c.flat(a[2], at::kFloat, R));
    g.top_k = static_cast<const int*>(c.flat(a[3], at::kInt, R));
    g.top_p = static_cast<const float*>(c.flat(a[4], at::kFloat, R));
    g.min_p = static_cast<const float*>(c.flat(a[5], at::kFloat, R));
    Tensor tokens, logprobs;
    if (a[6] == Py_None) {
        tokens = c.make({R}, at::kInt);
        g.tokens = tokens.data_ptr<int>();
    } else {
        g.tokens = static_cast<int*>(c.flat(a[6], at::kInt, R));
    }
    if (a[7] == Py_None) {
        logprobs = c.make({R}, at::kFloat);
        g.logprobs = logprobs.data_ptr<float>();
    } else {
        g.logprobs = static_cast<float*>(c.flat(a[7], at::kFloat, R));
    }
    if (!c.good || gala_sample(&g, c.stream(), nullptr, 0) < 0) Py_RETURN_NONE;
    PyObject* t = PyTuple_New(2);
    PyTuple_SET_ITEM(t, 0, wrap_or(a[6], tokens));
    PyTuple_SET_ITEM(t, 1, wrap_or(a[7], logprobs));
    return t;
    END
}

PyMethodDef methods[] = {
    {"layer_norm", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(layer_norm)), METH_FASTCALL, nullptr},
    {"gated_recurrence", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(gated_recurrence)), METH_FASTCALL, nullptr},
    {"gated_ffn", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(gated_ffn)), METH_FASTCALL, nullptr},
    {"sample", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(sample)), METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_front", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__front() {
    PyObject* m = PyModule_Create(&module);
    if (m && PyModule_AddStringConstant(m, "torch_version", GALA_TORCH_VERSION) < 0) Py_CLEAR(m);      // what it was compiled against
    return m;
}
