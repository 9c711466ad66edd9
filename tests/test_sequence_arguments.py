"""Refusals of the sequence-policy operators: what a call may not do is said before anything is enqueued, so no GPU is
needed.  Pointers are made-up addresses that nothing reads."""
import ctypes as C

import pytest

from paper_1906_04585_b200 import binding as B

P = 1 << 20


def refused(call, args, word, status=B.GALA_EINVAL):
    with pytest.raises(B.GalaError) as e:
        call(args)
    assert e.value.status == status and word in str(e.value), str(e.value)


def changed(make, **kw):
    a = make()
    for k, v in kw.items():
        assert hasattr(a, k)
        setattr(a, k, v)
    return a


def ln():
    return B.gala_layer_norm_args(B.GALA_BF16, B.GALA_BF16, 4, 32, 1e-5, P, 32, None, 0, P, P, P, 32, None, 0, P, P)


def ln_grad():
    return B.gala_layer_norm_grad_args(B.GALA_BF16, B.GALA_F32, 4, 32, P, 32, P, 32, None, 0, P, P, P, P, 32, P, P, P, 1 << 30)


def rec():
    return B.gala_recurrence_args(dtype=B.GALA_F32, steps=3, batch=2, dim=8, f=P, f_t=16, f_b=8, x=P, x_t=16, x_b=8, h=P, h_t=16, h_b=8)


def rec_grad():
    return B.gala_recurrence_grad_args(dtype=B.GALA_F32, steps=3, batch=2, dim=8, f=P, f_t=16, f_b=8, x=P, x_t=16, x_b=8, states=P, dh=P, dh_t=16,
                                       dh_b=8, df=P, df_t=16, df_b=8, dx=P, dx_t=16, dx_b=8)


def ffn():
    return B.gala_ffn_args(dtype=B.GALA_BF16, act=0, rows=4, dim=16, hidden=24, x=P, x_ld=16, w_gate=P, w_gate_ld=16, w_up=P, w_up_ld=16, w_down=P,
                           w_down_ld=24, y=P, y_ld=16, product=P, hidden_ld=24)


def ffn_grad():
    return B.gala_ffn_grad_args(dtype=B.GALA_BF16, act=0, rows=4, dim=16, hidden=24, dy=P, dy_ld=16, x=P, x_ld=16, w_gate=P, w_gate_ld=16, w_up=P,
                                w_up_ld=16, w_down=P, w_down_ld=24, product=P, gate=P, up=P, dgate=P, dup=P, hidden_ld=24, dx=P, dx_ld=16)


def draw():
    return B.gala_sample_args(B.GALA_F32, 3, 10, P, 10, P, None, None, None, None, P, None)


CASES = [
    (B.gala_layer_norm_forward, ln, dict(dtype=7), "dtype 7"),
    (B.gala_layer_norm_forward, ln, dict(wdtype=B.GALA_F16), "weights"),
    (B.gala_layer_norm_forward, ln, dict(cols=0), "columns"),
    (B.gala_layer_norm_forward, ln, dict(cols=16385, x_ld=16385, y_ld=16385), "16384"),
    (B.gala_layer_norm_forward, ln, dict(rows=-1), "-1 rows"),
    (B.gala_layer_norm_forward, ln, dict(eps=-1.0), "eps"),
    (B.gala_layer_norm_forward, ln, dict(eps=float("nan")), "eps"),
    (B.gala_layer_norm_forward, ln, dict(x=None), "needed"),
    (B.gala_layer_norm_forward, ln, dict(y_ld=31), "stride"),
    (B.gala_layer_norm_forward, ln, dict(residual=P, residual_ld=3), "stride"),
    (B.gala_layer_norm_forward, ln, dict(x=P + 1), "aligned"),
    (B.gala_layer_norm_forward, ln, dict(rstd=P + 2), "aligned"),
    (B.gala_layer_norm_backward, ln_grad, dict(dtype=3), "dtype 3"),
    (B.gala_layer_norm_backward, ln_grad, dict(dy=None), "needed"),
    (B.gala_layer_norm_backward, ln_grad, dict(dx_ld=1), "stride"),
    (B.gala_layer_norm_backward, ln_grad, dict(workspace=None), "workspace"),
    (B.gala_layer_norm_backward, ln_grad, dict(workspace_bytes=16), "workspace"),
    (B.gala_layer_norm_backward, ln_grad, dict(dweight=P + 2), "aligned"),
    (B.gala_gated_recurrence_forward, rec, dict(dtype=-1), "dtype"),
    (B.gala_gated_recurrence_forward, rec, dict(steps=-2), "negative"),
    (B.gala_gated_recurrence_forward, rec, dict(f=None), "needed"),
    (B.gala_gated_recurrence_forward, rec, dict(x=P + 2), "aligned"),
    (B.gala_gated_recurrence_forward, rec, dict(h_t=4), "overlap"),
    (B.gala_gated_recurrence_forward, rec, dict(h_b=0), "overlap"),
    (B.gala_gated_recurrence_forward, rec, dict(f_t=-16), "negative stride"),
    (B.gala_gated_recurrence_forward, rec, dict(x_t=1 << 30), "2^30"),
    (B.gala_gated_recurrence_forward, rec, dict(batch=1 << 40), "range"),
    (B.gala_gated_recurrence_forward, rec, dict(h0=P + 1), "float32"),
    (B.gala_gated_recurrence_backward, rec_grad, dict(states=None), "needed"),
    (B.gala_gated_recurrence_backward, rec_grad, dict(df_b=7), "overlap"),
    (B.gala_gated_recurrence_backward, rec_grad, dict(dh_t=1 << 30), "2^30"),
    (B.gala_gated_recurrence_backward, rec_grad, dict(dx=P + 1), "aligned"),
    (B.gala_gated_ffn_forward, ffn, dict(dtype=B.GALA_F32), "bfloat16 or float16"),
    (B.gala_gated_ffn_forward, ffn, dict(act=3), "act 3"),
    (B.gala_gated_ffn_forward, ffn, dict(dim=0), "dim 0"),
    (B.gala_gated_ffn_forward, ffn, dict(rows=1 << 31), "rows"),
    (B.gala_gated_ffn_forward, ffn, dict(x_ld=17), "multiple of 8"),
    (B.gala_gated_ffn_forward, ffn, dict(w_down_ld=16), "multiple of 8"),
    (B.gala_gated_ffn_forward, ffn, dict(w_up=P + 8), "16-byte"),
    (B.gala_gated_ffn_forward, ffn, dict(product=None), "16-byte"),
    (B.gala_gated_ffn_forward, ffn, dict(gate=P), "both or neither"),
    (B.gala_gated_ffn_backward, ffn_grad, dict(up=None), "16-byte"),
    (B.gala_gated_ffn_backward, ffn_grad, dict(dx_ld=20), "multiple of 8"),
    (B.gala_gated_ffn_backward, ffn_grad, dict(dw_up=P, dw_up_ld=8), "multiple of 8"),
    (B.gala_sample, draw, dict(dtype=9), "dtype 9"),
    (B.gala_sample, draw, dict(vocab=0), "entries"),
    (B.gala_sample, draw, dict(vocab=262145, logits_ld=262145), "262144"),
    (B.gala_sample, draw, dict(rows=1 << 27), "rows"),
    (B.gala_sample, draw, dict(uniforms=None), "needed"),
    (B.gala_sample, draw, dict(logits_ld=9), "stride"),
    (B.gala_sample, draw, dict(top_k=P + 2), "aligned"),
]


@pytest.mark.parametrize("call,make,change,word", CASES, ids=["%s-%s" % (c[0].__name__, "-".join(c[2])) for c in CASES])
def test_refusals(call, make, change, word):
    refused(call, changed(make, **change), word)


def test_null_arguments_and_short_messages():
    L = B.lib()
    for name in ("gala_layer_norm_forward", "gala_layer_norm_backward", "gala_gated_recurrence_forward", "gala_gated_recurrence_backward",
                 "gala_gated_ffn_forward", "gala_gated_ffn_backward", "gala_sample"):
        buf = C.create_string_buffer(b"x" * 12, 12)
        assert getattr(L, name)(None, None, buf, 12) == B.GALA_EINVAL
        assert buf.raw[11:] == b"\0" and buf.value == name[:11].encode()
        assert getattr(L, name)(None, None, None, 0) == B.GALA_EINVAL


def test_nothing_to_do_needs_no_device():
    B.gala_layer_norm_forward(changed(ln, rows=0, x=None, y=None))
    B.gala_gated_recurrence_forward(changed(rec, batch=0))
    B.gala_gated_recurrence_backward(changed(rec_grad, dim=0))
    B.gala_gated_ffn_forward(changed(ffn, rows=0))
    B.gala_sample(changed(draw, rows=0, logits=None))


def test_workspace():
    assert B.gala_layer_norm_workspace(0, 100) == 0
    assert B.gala_layer_norm_workspace(1 << 40, 16384) >= 2 * 16384 * 4
    with pytest.raises(B.GalaError):
        B.gala_layer_norm_workspace(4, 0)


def test_the_torch_front_end_wants_cuda_tensors():
    torch = pytest.importorskip("torch")
    from paper_1906_04585_b200 import sequence as S
    x = torch.zeros(4, 8)
    for call in (lambda: S.layer_norm(x), lambda: S.gated_recurrence(x.unsqueeze(0), x.unsqueeze(0)), lambda: S.gated_ffn(x, x, x, x.T),
                 lambda: S.sample(x, x[:, 0])):
        with pytest.raises(ValueError, match="CUDA"):
            call()
