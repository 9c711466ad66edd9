"""Refusals of the attention memory, the norm and rotation of queries and keys, and the adjustment of logits: what a call may
not do is said before anything is enqueued, so no GPU is needed.  Pointers are made-up addresses that nothing reads."""
import ctypes as C

import pytest

from paper_1906_04585_b200 import binding as B

P = 1 << 20


def changed(make, **kw):
    a = make()
    for k, v in kw.items():
        assert hasattr(a, k)
        setattr(a, k, v)
    return a


def attention(cls=None, **more):
    a = (cls or B.gala_linear_attention_args)()
    a.dtype, a.heads, a.dk, a.dv, a.steps, a.batch, a.scale, a.log_decay = B.GALA_BF16, 2, 8, 16, 3, 2, 1.0, P
    for n, w in (("q", 8), ("k", 8), ("v", 16)) + tuple(more.items()):
        setattr(a, n, P)
        setattr(a, n + "_t", 4 * w), setattr(a, n + "_b", 2 * w), setattr(a, n + "_h", w)
    a.workspace, a.workspace_bytes = P, 1 << 30
    return a


def forward():
    return attention(o=16)


def backward():
    return attention(B.gala_linear_attention_grad_args, grad_o=16, grad_q=8, grad_k=8, grad_v=16)


def qk(cls=B.gala_qk_norm_rotary_args, names=("q", "k", "q_out", "k_out")):
    a = cls()
    a.dtype, a.wdtype, a.q_heads, a.k_heads, a.dim, a.pairs, a.eps, a.tokens, a.positions, a.inv_freq = B.GALA_BF16, B.GALA_F32, 3, 2, 16, 8, 1e-6, 5, P, P
    for n in names:
        setattr(a, n, P), setattr(a, n + "_t", 48), setattr(a, n + "_h", 16)
    return a


def qk_grad():
    a = qk(B.gala_qk_norm_rotary_grad_args, ("q", "k", "grad_q_out", "grad_k_out", "grad_q", "grad_k"))
    a.grad_q_weight = a.grad_k_weight = a.workspace = P
    a.workspace_bytes = 1 << 30
    return a


def adjust():
    a = B.gala_adjust_logits_args()
    a.dtype, a.vocab, a.width, a.biases, a.rows, a.logits, a.logits_ld, a.out, a.out_ld = B.GALA_F32, 40, 7, 3, 4, P, 40, P, 40
    a.history, a.history_ld, a.bias_ids, a.bias_ids_ld, a.bias_values, a.bias_values_ld, a.mask, a.mask_ld = P, 7, P, 3, P, 3, P, 2
    return a


F, G, Q, R, A = B.gala_linear_attention_forward, B.gala_linear_attention_backward, B.gala_qk_norm_rotary_forward, B.gala_qk_norm_rotary_backward, B.gala_adjust_logits
CASES = [
    (F, forward, dict(dtype=3), "dtype 3"), (F, forward, dict(steps=-1), "range"), (F, forward, dict(steps=1 << 31), "range"),
    (F, forward, dict(batch=1 << 26), "range"), (F, forward, dict(heads=-2), "range"), (F, forward, dict(dk=129), "1 to 128"),
    (F, forward, dict(dv=0), "1 to 128"), (F, forward, dict(log_decay=None), "log_decay"), (F, forward, dict(log_decay=P + 1), "aligned"),
    (F, forward, dict(s0=P + 2), "aligned"), (F, forward, dict(s_last=P + 2), "aligned"), (F, forward, dict(status=P + 1), "aligned"),
    (F, forward, dict(k=None), "needed"), (F, forward, dict(v=P + 1), "aligned"), (F, forward, dict(q_t=-4), "negative"),
    (F, forward, dict(k_t=1 << 30), "2^30"), (F, forward, dict(v_h=1 << 35), "2^35"), (F, forward, dict(o=None), "o is needed"),
    (F, forward, dict(o=P + 1), "o is needed"), (F, forward, dict(o_h=15), "overlap"), (F, forward, dict(o_b=0), "overlap"), (F, forward, dict(o_t=63), "overlap"),
    (F, forward, dict(done=P, done_t=-1), "done"), (F, forward, dict(workspace=None, steps=500), "workspace"), (F, forward, dict(workspace=P + 8), "workspace"),
    (F, forward, dict(workspace_bytes=8, steps=500), "workspace"),
    (G, backward, dict(dtype=-1), "dtype"), (G, backward, dict(grad_o=None), "grad_o"), (G, backward, dict(grad_q=P + 1), "aligned"),
    (G, backward, dict(grad_k_h=7), "overlap"), (G, backward, dict(grad_v_t=1 << 30), "out of range"), (G, backward, dict(grad_s0=P + 1), "aligned"),
    (G, backward, dict(grad_o_b=-1), "negative"), (G, backward, dict(q=None), "needed"), (G, backward, dict(workspace=None, steps=500), "workspace"),
    (Q, qk, dict(dtype=5), "dtype 5"), (Q, qk, dict(wdtype=B.GALA_F16), "weights"), (Q, qk, dict(dim=257), "1 to 256"), (Q, qk, dict(pairs=9), "pairs"),
    (Q, qk, dict(pairs=-1), "pairs"), (Q, qk, dict(tokens=-1), "-1 tokens"), (Q, qk, dict(tokens=1 << 31), "tokens"), (Q, qk, dict(q_heads=65537), "heads"),
    (Q, qk, dict(eps=-1.0), "eps"), (Q, qk, dict(eps=float("nan")), "eps"), (Q, qk, dict(positions=None), "positions"), (Q, qk, dict(inv_freq=None), "inv_freq"),
    (Q, qk, dict(positions=P + 1), "aligned"), (Q, qk, dict(k_weight=P + 2), "aligned"), (Q, qk, dict(q=None), "needed"), (Q, qk, dict(k=P + 1), "needed"),
    (Q, qk, dict(q_t=-1), "negative"), (Q, qk, dict(k_h=1 << 32), "2^32"), (Q, qk, dict(q_out_h=15), "apart"), (Q, qk, dict(q_out_t=47), "apart"),
    (Q, qk, dict(k_out=None), "needed"),
    (R, qk_grad, dict(grad_q_out=None), "needed"), (R, qk_grad, dict(grad_k_h=0), "apart"), (R, qk_grad, dict(grad_q_weight=P + 2), "aligned"),
    (R, qk_grad, dict(workspace=None), "workspace"), (R, qk_grad, dict(workspace_bytes=100), "workspace"), (R, qk_grad, dict(dim=0), "1 to 256"),
    (A, adjust, dict(dtype=4), "dtype 4"), (A, adjust, dict(rows=-1), "rows"), (A, adjust, dict(rows=1 << 27), "rows"), (A, adjust, dict(vocab=0), "entries"),
    (A, adjust, dict(width=1 << 20), "2^20"), (A, adjust, dict(biases=4096), "4096"), (A, adjust, dict(biases=-1), "4096"), (A, adjust, dict(logits=None), "needed"),
    (A, adjust, dict(out=None), "needed"), (A, adjust, dict(logits=P + 2), "aligned"), (A, adjust, dict(bias_values=None), "bias_values"),
    (A, adjust, dict(logits_ld=39), "stride"), (A, adjust, dict(history_ld=6), "stride"), (A, adjust, dict(mask_ld=1), "stride"), (A, adjust, dict(bias_ids_ld=2), "stride"),
    (A, adjust, dict(mask=P + 1), "aligned"), (A, adjust, dict(frequency=P + 1), "aligned"),
]


@pytest.mark.parametrize("call,make,change,word", CASES, ids=["%s-%s-%d" % (c[0].__name__, "-".join(c[2]), i) for i, c in enumerate(CASES)])
def test_refusals(call, make, change, word):
    with pytest.raises(B.GalaError) as e:
        call(changed(make, **change))
    assert e.value.status == B.GALA_EINVAL and word in str(e.value), str(e.value)


def test_null_arguments_and_short_messages():
    L = B.lib()
    for name in ("gala_linear_attention_forward", "gala_linear_attention_backward", "gala_qk_norm_rotary_forward", "gala_qk_norm_rotary_backward",
                 "gala_adjust_logits"):
        buf = C.create_string_buffer(b"x" * 12, 12)
        assert getattr(L, name)(None, None, buf, 12) == B.GALA_EINVAL
        assert buf.raw[11:] == b"\0" and buf.value == name[:11].encode()
        assert getattr(L, name)(None, None, None, 0) == B.GALA_EINVAL


def test_nothing_to_do_needs_no_device():
    F(changed(forward, batch=0, q=None, log_decay=None))
    F(changed(forward, steps=0, q=None, o=None))
    G(changed(backward, heads=0, grad_o=None))
    Q(changed(qk, tokens=0, q=None))
    A(changed(adjust, rows=0, logits=None))


def test_workspaces():
    assert B.gala_linear_attention_workspace(0, 0, 0, 1, 1) >= 0
    assert B.gala_linear_attention_workspace(1 << 20, 1, 1, 128, 128) >= 128 * 128 * 4
    assert B.gala_qk_norm_rotary_workspace(0, 64) == 0 and B.gala_qk_norm_rotary_workspace(1, 64) >= 2 * 64 * 4
    for bad in ((-1, 1, 1, 8, 8), (1 << 31, 1, 1, 8, 8), (1, 1 << 27, 1, 8, 8), (1, 1, 1, 0, 8), (1, 1, 1, 8, 129)):
        with pytest.raises(B.GalaError):
            B.gala_linear_attention_workspace(*bad)
    with pytest.raises(B.GalaError):
        B.gala_qk_norm_rotary_workspace(4, 257)


def test_the_torch_front_end_wants_cuda_tensors():
    torch = pytest.importorskip("torch")
    from paper_1906_04585_b200 import sequence as S
    x = torch.zeros(4, 2, 3, 8)
    for call in (lambda: S.linear_attention(x, x, x, x[0, 0, :, 0]), lambda: S.linear_attention_backward(x, x, x, x, x[0, 0, :, 0]),
                 lambda: S.qk_norm_rotary(x[0], x[0], x[0, :, 0, 0].int(), x[0, 0, 0]),
                 lambda: S.qk_norm_rotary_backward(x[0], x[0], x[0], x[0], x[0, :, 0, 0].int(), x[0, 0, 0]), lambda: S.adjust_logits(x[0, 0])):
        with pytest.raises(ValueError, match="CUDA"):
            call()
