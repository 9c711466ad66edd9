"""Operators of sequence policies on torch tensors: layer norm, a gated linear recurrence over time, a gated
feed-forward block, and the draw of an action or token.

Argument checks and marshalling only, as in `learner`: every operator runs inside libgala.so (include/gala.h has the
formulas) on torch's current stream of the tensors' device, which has to be the current one.  Element types are float32,
bfloat16 and float16 (the feed-forward block: the 16-bit ones); states, statistics and log-probabilities are float32.
`out`-like arguments receive results in place; without them results are new tensors.  What a call may not do raises
GalaError (from the library) or TypeError / ValueError (from here) before anything is enqueued.

No call takes part in autograd: tensors that require gradients are read as they are, and results have no history.  The
backward passes are calls of their own.

Tensors that other streams still use have to be ordered by the caller, as with any torch operation.
"""
from __future__ import annotations

import importlib.util
import warnings
from typing import Optional

import torch

from . import binding as B

_DTYPE = {torch.float32: B.GALA_F32, torch.bfloat16: B.GALA_BF16, torch.float16: B.GALA_F16}
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (lambda index: torch.cuda.current_stream(index).cuda_stream)
_current_device = getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device

def _compiled():
    """The compiled front end, or None.  One that is there and cannot be used is worth a word: calls on small tensors take
    several times as long without it."""
    try:
        from . import _front
    except ImportError as e:
        if importlib.util.find_spec("._front", __package__) is not None:
            warnings.warn("the compiled front end does not load (%s): calls go through Python" % e)
        return None
    made, here = getattr(_front, "torch_version", "another one"), str(torch.__version__)
    if made != here:
        warnings.warn("the compiled front end is for torch %s, this is %s: calls go through Python until it is built again" % (made, here))
        return None
    return _front


# A call on small tensors is bound by the host.  The compiled front end (csrc/front.cpp) takes the forward calls whose
# arguments are as they should be; it returns None for all others, and the code below says what is wrong with them, or
# takes what only it can.  It is built with libgala.so where torch's headers are; without it every call goes through the
# code below.
_front = _compiled()


def _stream(t: torch.Tensor) -> int:
    if not t.is_cuda:
        raise ValueError("CUDA tensors are needed: there is no CPU fallback")
    index = t.get_device()
    if index != _current_device():
        raise ValueError("tensors are on %s, the current device is cuda:%d" % (t.device, torch.cuda.current_device()))
    return _raw_stream(index)


def _want(name: str, t: torch.Tensor, shape, dtype, like: torch.Tensor):
    if tuple(t.shape) != tuple(shape):
        raise ValueError("%s is %s, not %s" % (name, tuple(t.shape), tuple(shape)))
    if t.dtype != dtype:
        raise TypeError("%s is %s, not %s" % (name, t.dtype, dtype))
    if t.device != like.device:
        raise ValueError("%s is on %s, not on %s" % (name, t.device, like.device))


def _rows(name: str, t: Optional[torch.Tensor], shape, like: torch.Tensor):
    """Pointer and row stride of a matrix with contiguous columns (None: nothing)."""
    if t is None:
        return None, 0
    if t.is_contiguous() and t.dtype is like.dtype and t.shape == shape and t.get_device() == like.get_device() and shape[0] > 1:
        return t.data_ptr(), shape[1]
    _want(name, t, shape, like.dtype, like)
    if shape[1] > 1 and t.stride(1) != 1:
        raise ValueError("the columns of %s have to be contiguous" % name)
    # a single row may carry any stride: give it one that every operator takes
    return t.data_ptr(), t.stride(0) if shape[0] > 1 else (shape[1] + 7) // 8 * 8


def _flat(name: str, t: Optional[torch.Tensor], shape, dtype, like: torch.Tensor):
    """Pointer of a contiguous tensor (None: nothing)."""
    if t is None:
        return None
    if t.is_contiguous() and t.dtype is dtype and t.shape == shape and t.get_device() == like.get_device():
        return t.data_ptr()
    _want(name, t, shape, dtype, like)
    raise ValueError("%s has to be contiguous" % name)


def _type_of(t: torch.Tensor) -> int:
    try:
        return _DTYPE[t.dtype]
    except KeyError:
        raise TypeError("%s: float32, bfloat16 or float16 is needed" % t.dtype) from None


def _width(name: str, n: int) -> int:
    """A size that the library takes as a C int (which ctypes would cut to its low bits)."""
    if n >= 1 << 31:
        raise ValueError("%s is %d: too large" % (name, n))
    return n


_status = {}


def _status_word(t: torch.Tensor) -> int:
    index = t.get_device()
    if index not in _status:
        if torch.cuda.is_current_stream_capturing():
            return 0      # no word yet and no place to make one: this call goes without
        word = torch.zeros(1, dtype=torch.int32, device=t.device)
        torch.cuda.synchronize(index)      # streams that do not follow this one may use it next
        _status[index] = word, word.data_ptr()
    return _status[index][1]


def check() -> None:
    """Waits for the current stream and raises if a bounded wait inside a kernel of this module ran out since the last
    check (results since then are not to be trusted); the word is cleared.  Calls that were captured into a graph before
    the process's first call outside of one have no word to report to."""
    for word, _ in _status.values():
        if int(word.item()):
            word.zero_()
            raise B.GalaError(B.GALA_ECUDA, "a bounded device-side wait ran out")


# ---------------------------------------------------------------------------------------------- layer norm
def layer_norm(x: torch.Tensor, weight: Optional[torch.Tensor] = None, bias: Optional[torch.Tensor] = None, eps: float = 1e-5, *,
               residual: Optional[torch.Tensor] = None, out: Optional[torch.Tensor] = None, sum_out: Optional[torch.Tensor] = None):
    """Layer norm of s = x (+ residual) over its columns; x [rows, cols].  Returns (y, s, mean, rstd); s is x itself
    without a residual.  weight and bias [cols] are float32 or of x's type."""
    if _front is not None:
        done = _front.layer_norm(x, weight, bias, eps, residual, out, sum_out)
        if done is not None:
            return done
    st = _stream(x)
    if x.dim() != 2:
        raise ValueError("x has to be a matrix [rows, cols]")
    a = B.gala_layer_norm_args()
    a.dtype, shape = _type_of(x), x.shape
    a.rows, a.cols, a.eps = shape[0], _width("the number of columns", shape[1]), eps
    wdt = weight.dtype if weight is not None else bias.dtype if bias is not None else x.dtype
    a.wdtype = _DTYPE.get(wdt, -1)
    a.weight = _flat("weight", weight, shape[1:], wdt, x)
    a.bias = _flat("bias", bias, shape[1:], wdt, x)
    y = torch.empty(shape, dtype=x.dtype, device=x.device) if out is None else out
    a.x, a.x_ld = _rows("x", x, shape, x)
    a.y, a.y_ld = _rows("out", y, shape, x)
    s = x
    if residual is not None:
        s = torch.empty(shape, dtype=x.dtype, device=x.device) if sum_out is None else sum_out
        a.residual, a.residual_ld = _rows("residual", residual, shape, x)
        a.sum, a.sum_ld = _rows("sum_out", s, shape, x)
    elif sum_out is not None:
        raise ValueError("sum_out without residual")
    mean, rstd = torch.empty((2, shape[0]), dtype=torch.float32, device=x.device).unbind(0)
    a.mean, a.rstd = mean.data_ptr(), rstd.data_ptr()
    B.gala_layer_norm_forward(a, st)
    return y, s, mean, rstd


def layer_norm_backward(dy: torch.Tensor, x: torch.Tensor, mean: torch.Tensor, rstd: torch.Tensor, weight: Optional[torch.Tensor] = None, *,
                        dsum: Optional[torch.Tensor] = None, dx: Optional[torch.Tensor] = None, dweight: Optional[torch.Tensor] = None,
                        dbias: Optional[torch.Tensor] = None):
    """Gradients (dx, dweight, dbias) of layer_norm.  x: what was normalised (the s that layer_norm returned); dsum: the
    gradient that reaches s past the norm, added to dx, which is then the gradient of x and of the residual alike.
    dweight and dbias have weight's type (float32 without a weight)."""
    st = _stream(x)
    if x.dim() != 2:
        raise ValueError("x has to be a matrix [rows, cols]")
    a = B.gala_layer_norm_grad_args()
    a.dtype, shape = _type_of(x), x.shape
    a.rows, a.cols = shape[0], _width("the number of columns", shape[1])
    wdt = weight.dtype if weight is not None else torch.float32
    a.wdtype = _DTYPE.get(wdt, -1)
    dx = torch.empty(shape, dtype=x.dtype, device=x.device) if dx is None else dx
    dweight = torch.empty(shape[1], dtype=wdt, device=x.device) if dweight is None else dweight
    dbias = torch.empty(shape[1], dtype=wdt, device=x.device) if dbias is None else dbias
    a.dy, a.dy_ld = _rows("dy", dy, shape, x)
    a.x, a.x_ld = _rows("x", x, shape, x)
    a.dsum, a.dsum_ld = _rows("dsum", dsum, shape, x)
    a.dx, a.dx_ld = _rows("dx", dx, shape, x)
    a.mean = _flat("mean", mean, shape[:1], torch.float32, x)
    a.rstd = _flat("rstd", rstd, shape[:1], torch.float32, x)
    a.weight = _flat("weight", weight, shape[1:], wdt, x)
    a.dweight = _flat("dweight", dweight, shape[1:], wdt, x)
    a.dbias = _flat("dbias", dbias, shape[1:], wdt, x)
    a.workspace_bytes = B.gala_layer_norm_workspace(shape[0], shape[1])
    ws = torch.empty(a.workspace_bytes, dtype=torch.uint8, device=x.device)
    a.workspace = ws.data_ptr()
    B.gala_layer_norm_backward(a, st)
    return dx, dweight, dbias


# ---------------------------------------------------------------------------------------------- gated recurrence
def _steps(name: str, t: Optional[torch.Tensor], shape, dtype, like: torch.Tensor):
    """Pointer and the strides of time and sequence of a [steps, batch, dim] tensor with contiguous channels."""
    if t is None:
        return None, 0, 0
    if not (t.dtype is dtype and t.shape == shape and t.get_device() == like.get_device()):
        _want(name, t, shape, dtype, like)
    time, sequence, channel = t.stride()
    if channel != 1 and shape[2] > 1:
        raise ValueError("the channels of %s have to be contiguous" % name)
    return t.data_ptr(), time, sequence


def _done(done: Optional[torch.Tensor], shape, like: torch.Tensor):
    if done is None:
        return None, 0, 0
    if done.dtype not in (torch.uint8, torch.bool):
        raise TypeError("done is %s, not uint8 or bool" % done.dtype)
    _want("done", done, shape[:2], done.dtype, like)
    return done.data_ptr(), done.stride(0), done.stride(1)


def gated_recurrence(f: torch.Tensor, x: torch.Tensor, h0: Optional[torch.Tensor] = None, *, done: Optional[torch.Tensor] = None,
                     out: Optional[torch.Tensor] = None, h_last: Optional[torch.Tensor] = None, save: bool = False):
    """h_t = sigmoid(f_t) c_{t-1} + (1 - sigmoid(f_t)) x_t over time; c_t is h_t, or 0 where done_t; c_{-1} = h0.

    f, x [steps, batch, dim] with any strides for time and sequence (x.transpose(0, 1) for sequence-major data); done
    [steps, batch] with the meaning it has in a rollout.  Returns (h, h_last, states): h_last [batch, dim] is the h0 of
    the next call (pass the same tensor as h0 and h_last to keep a state in place), states is what the backward call
    needs (None unless `save`)."""
    if _front is not None and not save and x.is_cuda:
        got = _front.gated_recurrence(f, x, h0, done, out, h_last, _status_word(x))
        if got is not None:
            return got
    st = _stream(x)
    if x.dim() != 3:
        raise ValueError("x has to be [steps, batch, dim]")
    a = B.gala_recurrence_args()
    a.dtype, shape = _type_of(x), x.shape
    T, N, D = shape
    a.steps, a.batch, a.dim = T, N, D
    h = torch.empty(shape, dtype=x.dtype, device=x.device) if out is None else out
    h_last = torch.empty((N, D), dtype=torch.float32, device=x.device) if h_last is None else h_last
    states = torch.empty(((T + 7) // 8, N, D), dtype=torch.float32, device=x.device) if save else None
    a.f, a.f_t, a.f_b = _steps("f", f, shape, x.dtype, x)
    a.x, a.x_t, a.x_b = _steps("x", x, shape, x.dtype, x)
    a.h, a.h_t, a.h_b = _steps("out", h, shape, x.dtype, x)
    a.done, a.done_t, a.done_b = _done(done, shape, x)
    a.h0 = _flat("h0", h0, shape[1:], torch.float32, x)
    a.h_last = _flat("h_last", h_last, shape[1:], torch.float32, x)
    a.states = states.data_ptr() if save else None
    a.status = _status_word(x)
    B.gala_gated_recurrence_forward(a, st)
    return h, h_last, states


def gated_recurrence_backward(dh: Optional[torch.Tensor], f: torch.Tensor, x: torch.Tensor, states: torch.Tensor, *,
                              done: Optional[torch.Tensor] = None, dh_last: Optional[torch.Tensor] = None, df: Optional[torch.Tensor] = None,
                              dx: Optional[torch.Tensor] = None, dh0: Optional[torch.Tensor] = None):
    """Gradients (df, dx, dh0) of gated_recurrence from those of h (dh) and h_last (dh_last); states is the forward call's."""
    st = _stream(x)
    if x.dim() != 3:
        raise ValueError("x has to be [steps, batch, dim]")
    a = B.gala_recurrence_grad_args()
    a.dtype, shape = _type_of(x), x.shape
    T, N, D = shape
    a.steps, a.batch, a.dim = T, N, D
    df = torch.empty(shape, dtype=x.dtype, device=x.device) if df is None else df
    dx = torch.empty(shape, dtype=x.dtype, device=x.device) if dx is None else dx
    dh0 = torch.empty((N, D), dtype=torch.float32, device=x.device) if dh0 is None else dh0
    a.f, a.f_t, a.f_b = _steps("f", f, shape, x.dtype, x)
    a.x, a.x_t, a.x_b = _steps("x", x, shape, x.dtype, x)
    a.dh, a.dh_t, a.dh_b = _steps("dh", dh, shape, x.dtype, x)
    a.df, a.df_t, a.df_b = _steps("df", df, shape, x.dtype, x)
    a.dx, a.dx_t, a.dx_b = _steps("dx", dx, shape, x.dtype, x)
    a.done, a.done_t, a.done_b = _done(done, shape, x)
    a.states = _flat("states", states, ((T + 7) // 8, N, D), torch.float32, x)
    a.dh_last = _flat("dh_last", dh_last, shape[1:], torch.float32, x)
    a.dh0 = _flat("dh0", dh0, shape[1:], torch.float32, x)
    a.status = _status_word(x)
    B.gala_gated_recurrence_backward(a, st)
    return df, dx, dh0


# ---------------------------------------------------------------------------------------------- gated feed-forward
_ACT = {"silu": B.GALA_ACT_SILU, "gelu": B.GALA_ACT_GELU, "relu": B.GALA_ACT_RELU}
def _ffn_shapes(a, x, w_gate, w_up, w_down, act):
    if x.dim() != 2 or w_gate.dim() != 2:
        raise ValueError("x has to be [rows, dim], the weights [hidden, dim] and [dim, hidden]")
    rows, dim = x.shape
    hidden = w_gate.shape[0]
    try:
        a.act = _ACT[act]
    except KeyError:
        raise ValueError("activation %r: one of %s is needed" % (act, ", ".join(_ACT))) from None
    a.dtype, a.rows, a.dim, a.hidden = _type_of(x), rows, _width("dim", dim), _width("hidden", hidden)
    a.x, a.x_ld = _rows("x", x, (rows, dim), x)
    a.w_gate, a.w_gate_ld = _rows("w_gate", w_gate, (hidden, dim), x)
    a.w_up, a.w_up_ld = _rows("w_up", w_up, (hidden, dim), x)
    a.w_down, a.w_down_ld = _rows("w_down", w_down, (dim, hidden), x)
    a.hidden_ld = (hidden + 7) // 8 * 8
    a.status = _status_word(x)
    return rows, dim, hidden


def gated_ffn(x: torch.Tensor, w_gate: torch.Tensor, w_up: torch.Tensor, w_down: torch.Tensor, activation: str = "silu", *,
              out: Optional[torch.Tensor] = None, save: bool = False):
    """y = (act(x w_gate^T) * (x w_up^T)) w_down^T for x [rows, dim], w_gate and w_up [hidden, dim], w_down [dim, hidden],
    all bfloat16 or all float16; activation "silu", "gelu" or "relu".  Every matrix starts on a 16-byte boundary and has a
    row stride that is a multiple of 8.  Returns (y, saved); saved is what the backward call needs (None unless `save`)."""
    if _front is not None and not save and x.is_cuda:
        y = _front.gated_ffn(x, w_gate, w_up, w_down, _ACT.get(activation, -1), out, _status_word(x))
        if y is not None:
            return y, None
    st = _stream(x)
    a = B.gala_ffn_args()
    rows, dim, hidden = _ffn_shapes(a, x, w_gate, w_up, w_down, activation)
    if out is None:
        out = torch.empty((rows, (dim + 7) // 8 * 8), dtype=x.dtype, device=x.device)[:, :dim]
    a.y, a.y_ld = _rows("out", out, (rows, dim), x)
    kept = torch.empty((3 if save else 1, rows, a.hidden_ld), dtype=x.dtype, device=x.device)
    first, size = kept.data_ptr(), 2 * rows * a.hidden_ld
    a.product = first
    if save:
        a.gate, a.up = first + size, first + 2 * size
    B.gala_gated_ffn_forward(a, st)
    return out, kept if save else None


def gated_ffn_backward(dy: torch.Tensor, x: torch.Tensor, w_gate: torch.Tensor, w_up: torch.Tensor, w_down: torch.Tensor, saved: torch.Tensor,
                       activation: str = "silu", *, dx: Optional[torch.Tensor] = None, dw_gate: Optional[torch.Tensor] = None,
                       dw_up: Optional[torch.Tensor] = None, dw_down: Optional[torch.Tensor] = None):
    """Gradients (dx, dw_gate, dw_up, dw_down) of gated_ffn from dy [rows, dim]; saved is the forward call's."""
    st = _stream(x)
    a = B.gala_ffn_grad_args()
    rows, dim, hidden = _ffn_shapes(a, x, w_gate, w_up, w_down, activation)

    def grad(t, n, m):
        return torch.empty((n, (m + 7) // 8 * 8), dtype=x.dtype, device=x.device)[:, :m] if t is None else t

    dx, dw_gate, dw_up, dw_down = grad(dx, rows, dim), grad(dw_gate, hidden, dim), grad(dw_up, hidden, dim), grad(dw_down, dim, hidden)
    a.dy, a.dy_ld = _rows("dy", dy, (rows, dim), x)
    a.dx, a.dx_ld = _rows("dx", dx, (rows, dim), x)
    a.dw_gate, a.dw_gate_ld = _rows("dw_gate", dw_gate, (hidden, dim), x)
    a.dw_up, a.dw_up_ld = _rows("dw_up", dw_up, (hidden, dim), x)
    a.dw_down, a.dw_down_ld = _rows("dw_down", dw_down, (dim, hidden), x)
    first, size = _flat("saved", saved, (3, rows, a.hidden_ld), x.dtype, x), 2 * rows * a.hidden_ld
    a.product, a.gate, a.up = first, first + size, first + 2 * size
    work = torch.empty((2, rows, a.hidden_ld), dtype=x.dtype, device=x.device)
    first = work.data_ptr()
    a.dgate, a.dup = first, first + size
    B.gala_gated_ffn_backward(a, st)
    return dx, dw_gate, dw_up, dw_down


# ---------------------------------------------------------------------------------------------- drawing a token
def sample(logits: torch.Tensor, uniforms: torch.Tensor, temperature: Optional[torch.Tensor] = None, top_k: Optional[torch.Tensor] = None,
           top_p: Optional[torch.Tensor] = None, min_p: Optional[torch.Tensor] = None, *, out: Optional[torch.Tensor] = None,
           logprobs: Optional[torch.Tensor] = None):
    """One token a row of logits [rows, vocab], drawn by inverse CDF in the order of the index from the caller's uniforms
    [rows] in [0, 1) after temperature, top-k, top-p and min-p (each [rows] or None).  Returns (tokens int32, logprobs
    float32): the log-probability is that of the distribution that was drawn from.  Temperature <= 0 takes the largest
    entry; a row that is all -inf (or NaN) gives token -1."""
    if _front is not None:
        drawn = _front.sample(logits, uniforms, temperature, top_k, top_p, min_p, out, logprobs)
        if drawn is not None:
            return drawn
    st = _stream(logits)
    if logits.dim() != 2:
        raise ValueError("logits has to be a matrix [rows, vocab]")
    a = B.gala_sample_args()
    a.dtype, shape = _type_of(logits), logits.shape
    a.rows, a.vocab = shape[0], _width("the number of entries", shape[1])
    tokens = torch.empty(shape[0], dtype=torch.int32, device=logits.device) if out is None else out
    logprobs = torch.empty(shape[0], dtype=torch.float32, device=logits.device) if logprobs is None else logprobs
    a.logits, a.logits_ld = _rows("logits", logits, shape, logits)
    a.uniforms = _flat("uniforms", uniforms, shape[:1], torch.float32, logits)
    a.temperature = _flat("temperature", temperature, shape[:1], torch.float32, logits)
    a.top_k = _flat("top_k", top_k, shape[:1], torch.int32, logits)
    a.top_p = _flat("top_p", top_p, shape[:1], torch.float32, logits)
    a.min_p = _flat("min_p", min_p, shape[:1], torch.float32, logits)
    a.tokens = _flat("out", tokens, shape[:1], torch.int32, logits)
    a.logprobs = _flat("logprobs", logprobs, shape[:1], torch.float32, logits)
    B.gala_sample(a, st)
    return tokens, logprobs
