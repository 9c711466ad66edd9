"""GPU: argument checks of the torch front end of the attention memory, the norm and rotation of queries and keys and the
adjustment of logits, and their streams."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


def S():
    from paper_1906_04585_b200 import sequence
    return sequence


def t(*shape, dtype=torch.bfloat16):
    return torch.zeros(*shape, dtype=dtype, device="cuda")


def f(*shape):
    return t(*shape, dtype=torch.float32)


def i(*shape):
    return t(*shape, dtype=torch.int32)


def qkv(dk=8, dv=6, dtype=torch.bfloat16):
    return t(3, 2, 4, dk, dtype=dtype), t(3, 2, 4, dk, dtype=dtype), t(3, 2, 4, dv, dtype=dtype)


def memory(s, q=None, k=None, v=None, decay=None, *more, **named):
    a, b, c = qkv()
    return s.linear_attention(a if q is None else q, b if k is None else k, c if v is None else v, f(4) if decay is None else decay, *more, **named)


def norm(s, q=None, k=None, positions=None, freq=None, *more, **named):
    return s.qk_norm_rotary(t(5, 3, 8) if q is None else q, t(5, 2, 8) if k is None else k, i(5) if positions is None else positions,
                            f(4) if freq is None else freq, *more, **named)


BAD = [
    ("k of another width", ValueError, lambda s: memory(s, k=t(3, 2, 4, 9))),
    ("v of other steps", ValueError, lambda s: memory(s, v=t(2, 2, 4, 6))),
    ("v of another type", TypeError, lambda s: memory(s, v=t(3, 2, 4, 6, dtype=torch.float16))),
    ("q of a type it does not know", TypeError, lambda s: memory(s, *qkv(dtype=torch.float64))),
    ("q without a batch", ValueError, lambda s: memory(s, q=t(3, 4, 8))),
    ("q with strided channels", ValueError, lambda s: memory(s, q=t(3, 2, 8, 4).transpose(2, 3))),
    ("heads of 129", Exception, lambda s: memory(s, *qkv(129))),
    ("a decay too many", ValueError, lambda s: memory(s, decay=f(5))),
    ("a decay in 16 bits", TypeError, lambda s: memory(s, decay=t(4))),
    ("a decay on the CPU", ValueError, lambda s: memory(s, decay=torch.zeros(4))),
    ("a state in 16 bits", TypeError, lambda s: memory(s, None, None, None, None, t(2, 4, 8, 6))),
    ("a state the wrong way round", ValueError, lambda s: memory(s, None, None, None, None, f(2, 4, 6, 8))),
    ("done in 32 bits", TypeError, lambda s: memory(s, done=f(3, 2))),
    ("o whose rows overlap", Exception, lambda s: memory(s, out=t(1, 1, 1, 6).expand(3, 2, 4, 6))),
    ("gradients of o of another shape", ValueError, lambda s: s.linear_attention_backward(t(3, 2, 4, 8), *qkv(), f(4))),
    ("a gradient of the state in 16 bits", TypeError, lambda s: s.linear_attention_backward(t(3, 2, 4, 6), *qkv(), f(4), ds_last=t(2, 4, 8, 6))),
    ("keys of other tokens", ValueError, lambda s: norm(s, k=t(6, 2, 8))),
    ("keys of another type", TypeError, lambda s: norm(s, k=f(5, 2, 8))),
    ("queries that are a matrix", ValueError, lambda s: norm(s, q=t(5, 24))),
    ("queries with strided entries", ValueError, lambda s: norm(s, q=t(5, 8, 3).transpose(1, 2))),
    ("positions in 64 bits", TypeError, lambda s: norm(s, positions=t(5, dtype=torch.int64))),
    ("positions of other tokens", ValueError, lambda s: norm(s, positions=i(4))),
    ("more pairs than entries hold", Exception, lambda s: norm(s, freq=f(5))),
    ("frequencies in 16 bits", TypeError, lambda s: norm(s, freq=t(4))),
    ("a weight of another width", ValueError, lambda s: norm(s, None, None, None, None, f(9))),
    ("weights of two types", TypeError, lambda s: norm(s, None, None, None, None, f(8), t(8))),
    ("weights of a third type", Exception, lambda s: norm(s, None, None, None, None, t(8, dtype=torch.float16), t(8, dtype=torch.float16))),
    ("heads of 257", Exception, lambda s: norm(s, q=t(5, 3, 257), k=t(5, 2, 257))),
    ("a weight's gradient in 16 bits", TypeError, lambda s: s.qk_norm_rotary_backward(t(5, 3, 8), t(5, 2, 8), t(5, 3, 8), t(5, 2, 8), i(5), f(4), f(8), f(8), dq_weight=t(8))),
    ("logits of one row without its axis", ValueError, lambda s: s.adjust_logits(t(8))),
    ("logits with strided entries", ValueError, lambda s: s.adjust_logits(t(8, 4).T)),
    ("logits of a type it does not know", TypeError, lambda s: s.adjust_logits(t(4, 8, dtype=torch.float64))),
    ("history in 64 bits", TypeError, lambda s: s.adjust_logits(t(4, 8), history=t(4, 3, dtype=torch.int64))),
    ("history of other rows", ValueError, lambda s: s.adjust_logits(t(4, 8), history=i(5, 3))),
    ("lengths without a history", ValueError, lambda s: s.adjust_logits(t(4, 8), lengths=i(4))),
    ("a penalty without a history", ValueError, lambda s: s.adjust_logits(t(4, 8), presence=f(4))),
    ("a penalty for other rows", ValueError, lambda s: s.adjust_logits(t(4, 8), history=i(4, 3), repetition=f(3))),
    ("a penalty in 16 bits", TypeError, lambda s: s.adjust_logits(t(4, 8), history=i(4, 3), frequency=t(4))),
    ("biases without values", ValueError, lambda s: s.adjust_logits(t(4, 8), bias_ids=i(4, 2))),
    ("values without ids", ValueError, lambda s: s.adjust_logits(t(4, 8), bias_values=f(4, 2))),
    ("values of another width", ValueError, lambda s: s.adjust_logits(t(4, 8), bias_ids=i(4, 2), bias_values=f(4, 3))),
    ("4096 biases", Exception, lambda s: s.adjust_logits(t(4, 8), bias_ids=i(4, 4096), bias_values=f(4, 4096))),
    ("a mask of too few words", ValueError, lambda s: s.adjust_logits(t(4, 33), mask=i(4, 1))),
    ("a mask of truth values", Exception, lambda s: s.adjust_logits(t(4, 8), mask=t(4, 8, dtype=torch.bool))),
    ("out of another type", TypeError, lambda s: s.adjust_logits(t(4, 8), out=f(4, 8))),
    ("out whose rows overlap", Exception, lambda s: s.adjust_logits(t(4, 8), out=t(1, 8).expand(4, 8))),
]


@pytest.mark.parametrize("what,error,call", BAD, ids=[b[0].replace(" ", "-") for b in BAD])
def test_refuses(what, error, call):
    with pytest.raises(error):
        call(S())


def test_results_come_in_place_where_asked():
    q, k, v = (torch.randn(5, 2, 3, 8, device="cuda") for _ in range(3))
    decay, s = torch.full((3,), -0.1, device="cuda"), torch.randn(2, 3, 8, 8, device="cuda")
    want, last = S().linear_attention(q, k, v, decay, s.clone())
    out = torch.empty(5, 2, 3, 12, device="cuda")[..., :8]
    o, kept = S().linear_attention(q, k, v, decay, s, out=out, s_last=s)
    assert o is out and kept is s and torch.equal(o, want) and torch.equal(s, last)
    a, b = torch.randn(6, 3, 8, device="cuda"), torch.randn(6, 2, 8, device="cuda")
    pos, freq = torch.arange(6, dtype=torch.int32, device="cuda"), torch.rand(4, device="cuda")
    want = S().qk_norm_rotary(a, b, pos, freq)
    got = S().qk_norm_rotary(a, b, pos, freq, q_out=a, k_out=b)
    assert got[0] is a and got[1] is b and torch.equal(a, want[0]) and torch.equal(b, want[1])
    x, bias = torch.randn(4, 40, device="cuda"), torch.randn(4, 2, device="cuda")
    want = S().adjust_logits(x, bias_ids=i(4, 2), bias_values=bias)
    assert S().adjust_logits(x, bias_ids=i(4, 2), bias_values=bias, out=x) is x and torch.equal(x, want)


def calls(x, freq, pos, decay, hist, pen):
    """Each operator, on views of the one tensor x [512, 256]."""
    s = S()
    short, long, heads = x.view(4, 32, 4, 256)[..., :64], x.view(256, 1, 8, 64), x.view(512, 4, 64)
    out = [*s.linear_attention(short, short, short, decay[:4]), *s.linear_attention(long, long, long, decay),
           *s.linear_attention_backward(long, long, long, long, decay), *s.qk_norm_rotary(heads, heads, pos, freq),
           *s.qk_norm_rotary_backward(heads, heads, heads, heads, pos, freq)]
    return out + [s.adjust_logits(x, history=hist, presence=pen), s.adjust_logits(x.view(8, 16384), history=hist[:8], presence=pen[:8])]


def more():
    g = torch.Generator(device="cuda").manual_seed(1)
    x = torch.randn(512, 256, device="cuda", generator=g).bfloat16()
    return x, (torch.rand(32, device="cuda", generator=g), torch.arange(512, dtype=torch.int32, device="cuda"),
               torch.full((8,), -0.01, device="cuda"), torch.randint(0, 256, (512, 40), dtype=torch.int32, device="cuda", generator=g),
               torch.ones(512, device="cuda"))


def test_each_operator_follows_the_current_stream():
    """Work on a side stream behind a long copy on it: results are those of the finished inputs."""
    side, big = torch.cuda.Stream(), torch.randn(64 << 20, device="cuda")
    src, rest = more()
    want = calls(src, *rest)
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        x = torch.zeros_like(src)
        for _ in range(20):
            big.mul_(1.0)
        x.copy_(src)
        got = calls(x, *rest)
    side.synchronize()
    assert len(got) == len(want) and all(torch.equal(a, b) for a, b in zip(got, want))


def test_two_streams_at_once_and_two_graphs():
    """Calls on two streams, and two graphs replayed side by side, have workspaces of their own."""
    sides = [torch.cuda.Stream() for _ in range(2)]
    src, rest = more()
    inputs = [src, -2 * src]
    want = [calls(x, *rest) for x in inputs]
    torch.cuda.synchronize()
    got = [[], []]
    for _ in range(3):
        for n, side in enumerate(sides):
            with torch.cuda.stream(side):
                got[n] = calls(inputs[n], *rest)
    torch.cuda.synchronize()
    graphs, held = [], []
    for x in inputs:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            held.append(calls(x, *rest))
        graphs.append(g)
    for _ in range(3):
        for g, side in zip(graphs, sides):
            with torch.cuda.stream(side):
                g.replay()
    torch.cuda.synchronize()
    for n in range(2):
        assert all(torch.equal(a, b) for a, b in zip(got[n], want[n]))
        assert all(torch.equal(a, b) for a, b in zip(held[n], want[n]))


def test_first_use_inside_a_capture():
    """A process whose first call is captured: no word to report to is made there, and the graph replays."""
    import subprocess
    import sys
    code = ("import torch\n"
            "from paper_1906_04585_b200 import sequence as S\n"
            "q = torch.randn(300, 1, 2, 64, device='cuda').bfloat16(); d = torch.full((2,), -0.1, device='cuda'); o = torch.zeros_like(q)\n"
            "g = torch.cuda.CUDAGraph()\n"
            "with torch.cuda.graph(g):\n"
            "    S.linear_attention(q, q, q, d, out=o)\n"
            "g.replay(); torch.cuda.synchronize()\n"
            "assert torch.equal(o, S.linear_attention(q, q, q, d)[0])\n"
            "S.check()\n")
    r = subprocess.run([sys.executable, "-c", code], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stderr[-2000:]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["fp32", "bf16"])
@pytest.mark.parametrize("T", [0, 5, 100, 300, 1100])
def test_gradient_of_the_state_in_place(T, dtype):
    """ds0 takes the place of ds_last: the same gradients, whichever way a call of that length goes."""
    g = torch.Generator(device="cuda").manual_seed(T)
    do, q, k, v = (torch.randn(T, 2, 3, 64, device="cuda", generator=g).to(dtype) for _ in range(4))
    decay, s0, ds = torch.full((3,), -0.02, device="cuda"), *(torch.randn(2, 3, 64, 64, device="cuda", generator=g) for _ in range(2))
    want = S().linear_attention_backward(do, q, k, v, decay, s0, ds_last=ds.clone())
    got = S().linear_attention_backward(do, q, k, v, decay, s0, ds_last=ds, ds0=ds)
    assert got[3] is ds and all(torch.equal(a, b) for a, b in zip(got, want))
