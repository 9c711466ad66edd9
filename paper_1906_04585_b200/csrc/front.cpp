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

// [steps][batch][heads][width] with contiguous channels: pointer and the strides of time, sequence and head
void* heads_of(Call& c, const Tensor& t, int64_t T, int64_t N, int64_t H, int64_t W, long long& st, long long& sb, long long& sh) {
    if (t.dim() != 4 || t.size(0) != T || t.size(1) != N || t.size(2) != H || t.size(3) != W || (W > 1 && t.stride(3) != 1)) {
        c.good = false;
        return nullptr;
    }
    st = t.stride(0);
    sb = t.stride(1);
    sh = t.stride(2);
    return t.data_ptr();
}
void* heads_of(Call& c, PyObject* o, int64_t T, int64_t N, int64_t H, int64_t W, long long& st, long long& sb, long long& sh) {
    const Tensor* t = c.tensor(o, c.like.scalar_type());
    if (!t) {
        c.good = false;
        return nullptr;
    }
    return heads_of(c, *t, T, N, H, W, st, sb, sh);
}
// float32 [batch][heads][dk][dv], contiguous, or None
float* state_of(Call& c, PyObject* o, int64_t N, int64_t H, int64_t K, int64_t V) {
    const Tensor* t = c.tensor(o, at::kFloat);
    if (!t) return nullptr;
    if (t->dim() != 4 || t->size(0) != N || t->size(1) != H || t->size(2) != K || t->size(3) != V || !t->is_contiguous()) c.good = false;
    return c.good ? t->data_ptr<float>() : nullptr;
}
// What the forward and the backward call of the attention share: q, k, v, log_decay, s0, done, scale (a Python float), status.
template <typename A> bool attention_common(Call& c, A& g, PyObject* k, PyObject* v, PyObject* ld, PyObject* s0, PyObject* done, PyObject* scale, PyObject* status, Tensor& space) {
    const Tensor& q = c.like;
    g.dtype = type_of(q);
    if (!c.good || g.dtype < 0 || q.dim() != 4 || !THPVariable_Check(v) || THPVariable_Unpack(v).dim() != 4) return false;
    const int64_t T = q.size(0), N = q.size(1), H = q.size(2), K = q.size(3), V = THPVariable_Unpack(v).size(3);
    if (!fits(H) || !fits(K) || !fits(V)) return false;
    g.steps = T;
    g.batch = N;
    g.heads = (int)H;
    g.dk = (int)K;
    g.dv = (int)V;
    g.scale = (float)PyFloat_AsDouble(scale);
    g.status = static_cast<int*>(PyLong_AsVoidPtr(status));
    if (PyErr_Occurred()) return false;
    g.q = heads_of(c, q, T, N, H, K, g.q_t, g.q_b, g.q_h);
    g.k = heads_of(c, k, T, N, H, K, g.k_t, g.k_b, g.k_h);
    g.v = heads_of(c, v, T, N, H, V, g.v_t, g.v_b, g.v_h);
    g.log_decay = static_cast<const float*>(c.flat(ld, at::kFloat, H));
    g.s0 = state_of(c, s0, N, H, K, V);
    if (done != Py_None) {
        if (!THPVariable_Check(done)) return false;
        const at::ScalarType dt = THPVariable_Unpack(done).scalar_type();
        if (dt != at::kByte && dt != at::kBool) return false;
        const Tensor* d = c.tensor(done, dt);
        if (!d || d->dim() != 2 || d->size(0) != T || d->size(1) != N) return false;
        g.done = static_cast<const unsigned char*>(d->data_ptr());
        g.done_t = d->stride(0);
        g.done_b = d->stride(1);
    }
    if (!c.good) return false;
    g.workspace_bytes = gala_linear_attention_workspace(T, N, (int)H, (int)K, (int)V);
    if (g.workspace_bytes < 0) return false;
    space = c.make({g.workspace_bytes}, at::kByte);
    g.workspace = space.data_ptr();
    return true;
}

// linear_attention(q, k, v, log_decay, s0, done, scale, out, s_last, status)
PyObject* linear_attention(PyObject*, PyObject* const* a, Py_ssize_t n) {
    BEGIN
    if (n != 10 || !THPVariable_Check(a[0])) Py_RETURN_NONE;
    const Tensor& q = THPVariable_Unpack(a[0]);
    Call c(q);
    gala_linear_attention_args g = {};
    Tensor space, o, last;
    if (!attention_common(c, g, a[1], a[2], a[3], a[4], a[5], a[6], a[9], space)) {
        if (PyErr_Occurred()) return nullptr;
        Py_RETURN_NONE;
    }
    if (a[7] == Py_None) {
        o = c.make({g.steps, g.batch, g.heads, g.dv}, q.scalar_type());
        g.o = heads_of(c, o, g.steps, g.batch, g.heads, g.dv, g.o_t, g.o_b, g.o_h);
    } else {
        g.o = heads_of(c, a[7], g.steps, g.batch, g.heads, g.dv, g.o_t, g.o_b, g.o_h);
    }
    if (a[8] == Py_None) {
        last = c.make({g.batch, g.heads, g.dk, g.dv}, at::kFloat);
        g.s_last = last.data_ptr<float>();
    } else {
        g.s_last = state_of(c, a[8], g.batch, g.heads, g.dk, g.dv);
    }
    if (!c.good || gala_linear_attention_forward(&g, c.stream(), nullptr, 0) < 0) Py_RETURN_NONE;
    PyObject* t = PyTuple_New(2);
    PyTuple_SET_ITEM(t, 0, wrap_or(a[7], o));
    PyTuple_SET_ITEM(t, 1, wrap_or(a[8], last));
    return t;
    END
}

// linear_attention_backward(do, q, k, v, log_decay, s0, done, scale, ds_last, dq, dk, dv, ds0, status)
PyObject* linear_attention_backward(PyObject*, PyObject* const* a, Py_ssize_t n) {
    BEGIN
    if (n != 14 || !THPVariable_Check(a[1])) Py_RETURN_NONE;
    const Tensor& q = THPVariable_Unpack(a[1]);
    Call c(q);
    gala_linear_attention_grad_args g = {};
    Tensor space, dq, dk, dv, ds0;
    if (!attention_common(c, g, a[2], a[3], a[4], a[5], a[6], a[7], a[13], space)) {
        if (PyErr_Occurred()) return nullptr;
        Py_RETURN_NONE;
    }
    g.grad_o = heads_of(c, a[0], g.steps, g.batch, g.heads, g.dv, g.grad_o_t, g.grad_o_b, g.grad_o_h);
    g.grad_s_last = state_of(c, a[8], g.batch, g.heads, g.dk, g.dv);
    auto grad = [&](PyObject* given, Tensor& made, int64_t width, long long& st, long long& sb, long long& sh) {
        if (given != Py_None) return heads_of(c, given, g.steps, g.batch, g.heads, width, st, sb, sh);
        made = c.make({g.steps, g.batch, g.heads, width}, q.scalar_type());
        return heads_of(c, made, g.steps, g.batch, g.heads, width, st, sb, sh);
    };
    g.grad_q = grad(a[9], dq, g.dk, g.grad_q_t, g.grad_q_b, g.grad_q_h);
    g.grad_k = grad(a[10], dk, g.dk, g.grad_k_t, g.grad_k_b, g.grad_k_h);
    g.grad_v = grad(a[11], dv, g.dv, g.grad_v_t, g.grad_v_b, g.grad_v_h);
    if (a[12] == Py_None) {
        ds0 = c.make({g.batch, g.heads, g.dk, g.dv}, at::kFloat);
        g.grad_s0 = ds0.data_ptr<float>();
    } else {
        g.grad_s0 = state_of(c, a[12], g.batch, g.heads, g.dk, g.dv);
    }
    if (!c.good || gala_linear_attention_backward(&g, c.stream(), nullptr, 0) < 0) Py_RETURN_NONE;
    return four(wrap_or(a[9], dq), wrap_or(a[10], dk), wrap_or(a[11], dv), wrap_or(a[12], ds0));
    END
}

// [tokens][heads][dim] with contiguous entries
void* tokens_of(Call& c, const Tensor& t, int64_t N, int64_t H, int64_t D, long long& st, long long& sh) {
    if (t.dim() != 3 || t.size(0) != N || t.size(1) != H || t.size(2) != D || (D > 1 && t.stride(2) != 1)) {
        c.good = false;
        return nullptr;
    }
    st = t.stride(0);
    sh = t.stride(1);
    return t.data_ptr();
}
void* tokens_of(Call& c, PyObject* o, int64_t N, int64_t H, int64_t D, long long& st, long long& sh) {
    const Tensor* t = c.tensor(o, c.like.scalar_type());
    if (!t) {
        c.good = false;
        return nullptr;
    }
    return tokens_of(c, *t, N, H, D, st, sh);
}
// What the forward and the backward call share: q, k, positions, inv_freq, q_weight, k_weight, eps, interleaved; the weights' type
template <typename A> bool norm_common(Call& c, A& g, PyObject* const* a, at::ScalarType& wt) {
    const Tensor& q = c.like;
    g.dtype = type_of(q);
    if (!c.good || g.dtype < 0 || q.dim() != 3 || !THPVariable_Check(a[1]) || THPVariable_Unpack(a[1]).dim() != 3 || !THPVariable_Check(a[3])) return false;
    const int64_t N = q.size(0), HQ = q.size(1), D = q.size(2), HK = THPVariable_Unpack(a[1]).size(1);
    const Tensor& f = THPVariable_Unpack(a[3]);
    if (f.dim() != 1 || !fits(HQ) || !fits(HK) || !fits(D) || !fits(f.size(0))) return false;
    wt = at::kFloat;
    for (int i = 5; i > 3; i--)
        if (THPVariable_Check(a[i])) wt = THPVariable_Unpack(a[i]).scalar_type();
    g.wdtype = wt == at::kFloat ? (int)GALA_F32 : wt == q.scalar_type() ? g.dtype : -1;
    g.tokens = N;
    g.q_heads = (int)HQ;
    g.k_heads = (int)HK;
    g.dim = (int)D;
    g.pairs = (int)f.size(0);
    g.eps = (float)PyFloat_AsDouble(a[6]);
    g.interleaved = PyObject_IsTrue(a[7]);
    if (PyErr_Occurred()) return false;
    g.q = tokens_of(c, q, N, HQ, D, g.q_t, g.q_h);
    g.k = tokens_of(c, a[1], N, HK, D, g.k_t, g.k_h);
    g.positions = static_cast<const int*>(c.flat(a[2], at::kInt, N));
    g.inv_freq = static_cast<const float*>(c.flat(a[3], at::kFloat, f.size(0)));
    g.q_weight = c.flat(a[4], wt, D);
    g.k_weight = c.flat(a[5], wt, D);
    return c.good;
}

// qk_norm_rotary(q, k, positions, inv_freq, q_weight, k_weight, eps, interleaved, q_out, k_out)
PyObject* qk_norm_rotary(PyObject*, PyObject* const* a, Py_ssize_t n) {
    BEGIN
    if (n != 10 || !THPVariable_Check(a[0])) Py_RETURN_NONE;
    const Tensor& q = THPVariable_Unpack(a[0]);
    Call c(q);
    gala_qk_norm_rotary_args g = {};
    at::ScalarType wt;
    if (!norm_common(c, g, a, wt)) {
        if (PyErr_Occurred()) return nullptr;
        Py_RETURN_NONE;
    }
    Tensor qo, ko;
    auto out = [&](PyObject* given, Tensor& made, int64_t heads, long long& st, long long& sh) {
        if (given != Py_None) return tokens_of(c, given, g.tokens, heads, g.dim, st, sh);
        made = c.make({g.tokens, heads, g.dim}, q.scalar_type());
        return tokens_of(c, made, g.tokens, heads, g.dim, st, sh);
    };
    g.q_out = out(a[8], qo, g.q_heads, g.q_out_t, g.q_out_h);
    g.k_out = out(a[9], ko, g.k_heads, g.k_out_t, g.k_out_h);
    if (!c.good || gala_qk_norm_rotary_forward(&g, c.stream(), nullptr, 0) < 0) Py_RETURN_NONE;
    PyObject* t = PyTuple_New(2);
    PyTuple_SET_ITEM(t, 0, wrap_or(a[8], qo));
    PyTuple_SET_ITEM(t, 1, wrap_or(a[9], ko));
    return t;
    END
}

// qk_norm_rotary_backward(q, k, positions, inv_freq, q_weight, k_weight, eps, interleaved, dq_out, dk_out, dq, dk, dq_weight, dk_weight)
PyObject* qk_norm_rotary_backward(PyObject*, PyObject* const* a, Py_ssize_t n) {
    BEGIN
    if (n != 14 || !THPVariable_Check(a[0])) Py_RETURN_NONE;
    const Tensor& q = THPVariable_Unpack(a[0]);
    Call c(q);
    gala_qk_norm_rotary_grad_args g = {};
    at::ScalarType wt;
    if (!norm_common(c, g, a, wt)) {
        if (PyErr_Occurred()) return nullptr;
        Py_RETURN_NONE;
    }
    Tensor dq, dk, dwq, dwk;
    g.grad_q_out = tokens_of(c, a[8], g.tokens, g.q_heads, g.dim, g.grad_q_out_t, g.grad_q_out_h);
    g.grad_k_out = tokens_of(c, a[9], g.tokens, g.k_heads, g.dim, g.grad_k_out_t, g.grad_k_out_h);
    auto out = [&](PyObject* given, Tensor& made, int64_t heads, long long& st, long long& sh) {
        if (given != Py_None) return tokens_of(c, given, g.tokens, heads, g.dim, st, sh);
        made = c.make({g.tokens, heads, g.dim}, q.scalar_type());
        return tokens_of(c, made, g.tokens, heads, g.dim, st, sh);
    };
    g.grad_q = out(a[10], dq, g.q_heads, g.grad_q_t, g.grad_q_h);
    g.grad_k = out(a[11], dk, g.k_heads, g.grad_k_t, g.grad_k_h);
    auto weight = [&](PyObject* given, Tensor& made) {
        if (given != Py_None) return c.flat(given, wt, g.dim);
        made = c.make({g.dim}, wt);
        return made.data_ptr();
    };
    g.grad_q_weight = weight(a[12], dwq);
    g.grad_k_weight = weight(a[13], dwk);
    if (!c.good) Py_RETURN_NONE;
    g.workspace_bytes = gala_qk_norm_rotary_workspace(g.tokens, g.dim);
    if (g.workspace_bytes < 0) Py_RETURN_NONE;
    const Tensor space = c.make({g.workspace_bytes}, at::kByte);
    g.workspace = space.data_ptr();
    if (gala_qk_norm_rotary_backward(&g, c.stream(), nullptr, 0) < 0) Py_RETURN_NONE;
    return four(wrap_or(a[10], dq), wrap_or(a[11], dk), wrap_or(a[12], dwq), wrap_or(a[13], dwk));
    END
}

// adjust_logits(logits, history, lengths, repetition, frequency, presence, bias_ids, bias_values, mask, out)
PyObject* adjust_logits(PyObject*, PyObject* const* a, Py_ssize_t n) {
    BEGIN
    if (n != 10 || !THPVariable_Check(a[0])) Py_RETURN_NONE;
    const Tensor& l = THPVariable_Unpack(a[0]);
    Call c(l);
    gala_adjust_logits_args g = {};
    g.dtype = type_of(l);
    if (!c.good || g.dtype < 0 || l.dim() != 2) Py_RETURN_NONE;
    const int64_t R = l.size(0), V = l.size(1);
    if (!fits(V)) Py_RETURN_NONE;
    g.rows = R;
    g.vocab = (int)V;
    g.logits = c.rows(l, R, V, g.logits_ld);
    // a matrix of 32-bit numbers with contiguous columns; its number of columns where `width` is negative
    auto matrix = [&](PyObject* o, at::ScalarType type, int64_t rows, int64_t& width, long long& ld) -> void* {
        const Tensor* t = c.tensor(o, type);
        if (!t) return nullptr;
        if (t->dim() != 2 || t->size(0) != rows || (width >= 0 && t->size(1) != width) || !fits(t->size(1)) || (t->size(1) > 1 && t->stride(1) != 1)) {
            c.good = false;
            return nullptr;
        }
        width = t->size(1);
        ld = rows > 1 ? t->stride(0) : width;
        return t->data_ptr();
    };
    if (a[1] != Py_None) {
        int64_t width = -1;
        g.history = static_cast<const int*>(matrix(a[1], at::kInt, R, width, g.history_ld));
        g.width = (int)width;
        g.lengths = static_cast<const int*>(c.flat(a[2], at::kInt, R));
        g.repetition = static_cast<const float*>(c.flat(a[3], at::kFloat, R));
        g.frequency = static_cast<const float*>(c.flat(a[4], at::kFloat, R));
        g.presence = static_cast<const float*>(c.flat(a[5], at::kFloat, R));
    } else {
        for (int i = 2; i < 6; i++)
            if (a[i] != Py_None) Py_RETURN_NONE;
    }
    if ((a[6] == Py_None) != (a[7] == Py_None)) Py_RETURN_NONE;
    if (a[6] != Py_None) {
        int64_t width = -1;
        g.bias_ids = static_cast<const int*>(matrix(a[6], at::kInt, R, width, g.bias_ids_ld));
        g.biases = (int)width;
        g.bias_values = static_cast<const float*>(matrix(a[7], at::kFloat, R, width, g.bias_values_ld));
    }
    if (a[8] != Py_None) {
        if (!THPVariable_Check(a[8])) Py_RETURN_NONE;
        int64_t words = (V + 31) / 32;
        const Tensor& m = THPVariable_Unpack(a[8]);
        const bool shared = m.dim() == 2 && m.size(0) == 1;
        g.mask = static_cast<const int*>(matrix(a[8], at::kInt, shared ? 1 : R, words, g.mask_ld));
        if (shared) g.mask_ld = 0;
    }
    Tensor out;
    if (a[9] == Py_None) {
        out = c.make({R, V}, l.scalar_type());
        g.out = c.rows(out, R, V, g.out_ld);
    } else {
        g.out = c.rows(a[9], R, V, g.out_ld);
    }
    if (!c.good || gala_adjust_logits(&g, c.stream(), nullptr, 0) < 0) Py_RETURN_NONE;
    return wrap_or(a[9], out);
    END
}

PyMethodDef methods[] = {
    {"layer_norm", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(layer_norm)), METH_FASTCALL, nullptr},
    {"gated_recurrence", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(gated_recurrence)), METH_FASTCALL, nullptr},
    {"gated_ffn", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(gated_ffn)), METH_FASTCALL, nullptr},
    {"sample", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(sample)), METH_FASTCALL, nullptr},
    {"linear_attention", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(linear_attention)), METH_FASTCALL, nullptr},
    {"linear_attention_backward", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(linear_attention_backward)), METH_FASTCALL, nullptr},
    {"qk_norm_rotary", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(qk_norm_rotary)), METH_FASTCALL, nullptr},
    {"qk_norm_rotary_backward", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(qk_norm_rotary_backward)), METH_FASTCALL, nullptr},
    {"adjust_logits", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(adjust_logits)), METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_front", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__front() {
    PyObject* m = PyModule_Create(&module);
    if (m && PyModule_AddStringConstant(m, "torch_version", GALA_TORCH_VERSION) < 0) Py_CLEAR(m);      // what it was compiled against
    return m;
}
