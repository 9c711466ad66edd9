"""GPU: argument checks of the torch front end of the sequence-policy operators, and its streams."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


def S():
    from paper_1906_04585_b200 import sequence
    return sequence


def t(*shape, dtype=torch.bfloat16):
    return torch.zeros(*shape, dtype=dtype, device="cuda")


BAD = [
    ("weight of another width", ValueError, lambda s: s.layer_norm(t(4, 8), t(9))),
    ("bias of another type than the weight", TypeError, lambda s: s.layer_norm(t(4, 8), t(8), t(8, dtype=torch.float32))),
    ("weights of a third type", Exception, lambda s: s.layer_norm(t(4, 8), t(8, dtype=torch.float16))),
    ("x with strided columns", ValueError, lambda s: s.layer_norm(t(8, 4).T)),
    ("x of a type it does not know", TypeError, lambda s: s.layer_norm(t(4, 8, dtype=torch.float64))),
    ("x that is no matrix", ValueError, lambda s: s.layer_norm(t(8))),
    ("residual of another type", TypeError, lambda s: s.layer_norm(t(4, 8), residual=t(4, 8, dtype=torch.float32))),
    ("sum_out without residual", ValueError, lambda s: s.layer_norm(t(4, 8), sum_out=t(4, 8))),
    ("out on the CPU", ValueError, lambda s: s.layer_norm(t(4, 8), out=torch.zeros(4, 8, dtype=torch.bfloat16))),
    ("f of another shape", ValueError, lambda s: s.gated_recurrence(t(3, 2, 8), t(3, 2, 9))),
    ("h0 in 16 bits", TypeError, lambda s: s.gated_recurrence(t(3, 2, 8), t(3, 2, 8), t(2, 8))),
    ("done in 32 bits", TypeError, lambda s: s.gated_recurrence(t(3, 2, 8), t(3, 2, 8), done=t(3, 2, dtype=torch.float32))),
    ("x with strided channels", ValueError, lambda s: s.gated_recurrence(t(3, 2, 8), t(3, 8, 2).transpose(1, 2))),
    ("out whose rows overlap", Exception, lambda s: s.gated_recurrence(t(3, 2, 8), t(3, 2, 8), out=t(1, 1, 8).expand(3, 2, 8))),
    ("states of another length", ValueError, lambda s: s.gated_recurrence_backward(None, t(9, 2, 8), t(9, 2, 8), t(1, 2, 8, dtype=torch.float32))),
    ("float32 weights", Exception, lambda s: s.gated_ffn(*(t(8, 8, dtype=torch.float32) for _ in range(4)))),
    ("an activation it does not know", ValueError, lambda s: s.gated_ffn(t(2, 8), t(8, 8), t(8, 8), t(8, 8), "tanh")),
    ("w_down the wrong way round", ValueError, lambda s: s.gated_ffn(t(2, 8), t(16, 8), t(16, 8), t(16, 8))),
    ("rows that are not 16-byte aligned", Exception, lambda s: s.gated_ffn(t(2, 12), t(8, 12), t(8, 12), t(12, 8))),
    ("uniforms in 64 bits", TypeError, lambda s: s.sample(t(2, 8), t(2, dtype=torch.float64))),
    ("temperature for other rows", ValueError, lambda s: s.sample(t(2, 8), t(2, dtype=torch.float32), t(3, dtype=torch.float32))),
    ("top_k in 64 bits", TypeError, lambda s: s.sample(t(2, 8), t(2, dtype=torch.float32), None, t(2, dtype=torch.int64))),
    ("logits without entries", Exception, lambda s: s.sample(t(2, 0), t(2, dtype=torch.float32))),
    ("tokens in 64 bits", TypeError, lambda s: s.sample(t(2, 8), t(2, dtype=torch.float32), out=t(2, dtype=torch.int64))),
]


@pytest.mark.parametrize("what,error,call", BAD, ids=[b[0].replace(" ", "-") for b in BAD])
def test_refuses(what, error, call):
    with pytest.raises(error):
        call(S())


def test_results_come_in_place_where_asked():
    x, w = torch.randn(6, 40, device="cuda"), torch.randn(40, device="cuda")
    out, total = torch.empty(6, 48, device="cuda")[:, :40], torch.empty_like(x)
    y, s, mean, rstd = S().layer_norm(x, w, w, residual=x, out=out, sum_out=total)
    assert y.data_ptr() == out.data_ptr() and s is total and torch.equal(s, 2 * x)
    h, h0 = torch.empty(5, 6, 8, device="cuda"), torch.randn(6, 8, device="cuda")
    f = torch.randn(5, 6, 16, device="cuda")
    got, last, states = S().gated_recurrence(f[..., :8], f[..., 8:], h0, out=h, h_last=h0)
    assert got is h and last is h0 and states is None and torch.equal(h[-1], h0)
    tok, lp = torch.empty(6, dtype=torch.int32, device="cuda"), torch.empty(6, device="cuda")
    a, b = S().sample(x, torch.rand(6, device="cuda"), out=tok, logprobs=lp)
    assert a is tok and b is lp


def test_each_operator_follows_the_current_stream():
    """Work on a side stream behind a long copy on it: results are those of the finished inputs."""
    side = torch.cuda.Stream()
    big = torch.randn(64 << 20, device="cuda")
    src = torch.randn(512, 256, device="cuda", generator=torch.Generator(device="cuda").manual_seed(1)).bfloat16()
    w = torch.randn(256, 256, device="cuda").bfloat16() / 16
    u = torch.rand(512, device="cuda")
    want = (S().layer_norm(src)[0], S().gated_recurrence(src.view(8, 64, 256), src.view(8, 64, 256))[0], S().gated_ffn(src, w, w, w)[0], S().sample(src, u)[0])
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        x = torch.zeros_like(src)
        for _ in range(20):
            big.mul_(1.0)
        x.copy_(src)
        got = (S().layer_norm(x)[0], S().gated_recurrence(x.view(8, 64, 256), x.view(8, 64, 256))[0], S().gated_ffn(x, w, w, w)[0], S().sample(x, u)[0])
    side.synchronize()
    for a, b in zip(got, want):
        assert torch.equal(a, b)


def test_a_single_row_may_carry_any_stride():
    wide = torch.randn(1, 45, device="cuda").bfloat16()
    w = (torch.randn(24, 16, device="cuda") / 4).bfloat16()[:, :12]
    wd = (torch.randn(12, 24, device="cuda") / 4).bfloat16()
    x = wide[:, :12]
    y, saved = S().gated_ffn(x, w, w, wd, save=True)
    assert torch.equal(y, S().gated_ffn(x, w, w, wd)[0])
    padded = torch.zeros(2, 16, device="cuda", dtype=torch.bfloat16)
    padded[:1, :12] = x
    assert torch.equal(y, S().gated_ffn(padded[:, :12], w, w, wd)[0][:1])
    S().gated_ffn_backward(y, x, w, w, wd, saved)
    assert torch.equal(S().layer_norm(x)[0], S().layer_norm(padded[:, :12])[0][:1])
    assert int(S().sample(x, torch.zeros(1, device="cuda"))[0]) == 0


def test_first_use_inside_a_capture():
    """A process whose first call is captured: no word to report to is made there, and the graph replays."""
    import subprocess
    import sys
    code = ("import torch\n"
            "from paper_1906_04585_b200 import sequence as S\n"
            "f = torch.randn(40, 2, 64, device='cuda'); x = torch.randn(40, 2, 64, device='cuda'); h = torch.zeros_like(x)\n"
            "g = torch.cuda.CUDAGraph()\n"
            "with torch.cuda.graph(g):\n"
            "    S.gated_recurrence(f, x, out=h)\n"
            "g.replay(); torch.cuda.synchronize()\n"
            "assert torch.equal(h, S.gated_recurrence(f, x)[0])\n"
            "S.check()\n")
    r = subprocess.run([sys.executable, "-c", code], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stderr[-2000:]
