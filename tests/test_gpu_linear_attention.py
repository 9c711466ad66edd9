"""GPU: attention with a memory of fixed size, forward and backward, against a step-by-step evaluation in 64 bits.

Bounds come from a running analysis beside the 64-bit evaluation.  eps = 2^-24, u = half a step of the element type.  Beside
the state X runs its absolute sum A (every product taken positive) and E, three roundings of A a step (the product, the sum,
the fade) faded along with it: what a sequential float32 evaluation is off by.  Joining pieces of the time axis passes through
the same sums once more, hence 2 E.  An output sums dk products: (dk + 8) eps of the absolute sum.

In 16 bits a long call goes through tensor cores by chunks.  Scores and the state are then rounded to the element type as
operands (every term of an output passes one of the two: u, and the scores' own float32 sums of dk terms), the weighted values
that add to the state are held in two pieces (u^2), and sums of 128 terms are taken in float32 without a known order; a fade
over n steps is one exponential, off by |n log_decay| + 2 roundings, less than 4 of the absolute sum where it is not small.
So: outputs (u + u^2 + (dk + 300) eps) of the absolute sum, states (u^2 + 300 eps).
"""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

EPS = 2.0 ** -24
U = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}


def S():
    from paper_1906_04585_b200 import sequence
    return sequence


class Pass:
    """One pass: X = gain X + k v^T, o = X^T q, with the running bounds, step by step; link[p]: whether what was held before
    step p is dropped."""

    def __init__(self, q, k, v, log_decay, link, first, entry):
        q, k, v = q.double(), k.double(), v.double()
        T, N, H, dk = q.shape
        dv = v.shape[-1]
        g = torch.exp(log_decay.double().clamp(max=0)).view(1, H, 1, 1)
        X = torch.zeros(N, H, dk, dv, dtype=torch.float64, device=q.device) if first is None else first.double()
        A, E = X.abs(), torch.zeros_like(X)
        self.o, self.a, self.e = (torch.zeros(T, N, H, dv, dtype=torch.float64, device=q.device) for _ in range(3))
        for t in range(T):
            gain = torch.ones_like(g) if t == 0 and not entry else g
            if link is not None:
                drop = link[t].view(N, 1, 1, 1)
                X, A, E = (torch.where(drop, 0.0, x) for x in (X, A, E))
            kv = k[t].unsqueeze(-1) * v[t].unsqueeze(-2)
            X = gain * X + kv
            A = gain * A + kv.abs()
            E = gain * E + 3 * EPS * A
            self.o[t] = (q[t].unsqueeze(-1) * X).sum(-2)
            self.a[t] = (q[t].abs().unsqueeze(-1) * A).sum(-2)
            self.e[t] = (q[t].abs().unsqueeze(-1) * E).sum(-2)
        self.X, self.A, self.E = X, A, E


def check(name, got, want, absolute, running, width, dtype, state=False):
    u = U[dtype]
    chunk = 0.0 if dtype == torch.float32 else (u * u + 300 * EPS if state else u + u * u + 300 * EPS)
    bound = (0.0 if state else u) * want.abs() + EPS * want.abs() + 2 * running + (chunk + (width + 8) * EPS) * absolute * (1 + u) + 1e-37
    if dtype == torch.float16:
        bound = bound + (0.0 if state else 2.0 ** -25) + (1e-6 if not state else 0.0) * absolute      # numbers below 2^-14 have fewer digits
    off = (got.double() - want).abs()
    # a value past the type's largest number (by less than half a step it is still rounded to it) is infinite there
    past = torch.isinf(got) & (got.double().sign() == want.sign()) & (want.abs() + bound > torch.finfo(got.dtype).max)
    bad = ~(off <= bound) & ~past
    assert not bad.any(), "%s: %d of %d outside, worst %.3g times the bound" % (name, int(bad.sum()), bad.numel(), float((off / bound)[bad].max()))


def check_all(q, k, v, ld, s0, done, scale, do=None, ds_last=None, got=None, got_grad=None):
    dtype, T, dk, dv = q.dtype, q.shape[0], q.shape[-1], v.shape[-1]
    cut = None if done is None else done != 0
    before = None if cut is None else torch.cat([torch.zeros_like(cut[:1]), cut[:-1]])
    if got is not None:
        p = Pass(q, k, v, ld, before, s0, True)
        check("o", got[0], scale * p.o, scale * p.a, scale * p.e, dk, dtype)
        keep = torch.ones_like(p.X) if cut is None else (~cut[-1]).double().view(-1, 1, 1, 1)
        check("s_last", got[1], keep * p.X, keep * p.A, keep * p.E, 0, dtype, state=True)
    if got_grad is not None:
        def t(x):
            return None if x is None else x.transpose(-1, -2)

        def f(x):
            return None if x is None else x.flip(0)

        p = Pass(do, v, k, ld, before, t(s0), True)
        check("dq", got_grad[0], scale * p.o, scale * p.a, scale * p.e, dv, dtype)
        p = Pass(f(v), scale * f(do).double(), f(q), ld, f(cut), t(ds_last), False)
        check("dk", got_grad[1], f(p.o), f(p.a), f(p.e), dv, dtype)
        p = Pass(f(k), f(q), scale * f(do).double(), ld, f(cut), ds_last, False)
        check("dv", got_grad[2], f(p.o), f(p.a), f(p.e), dk, dtype)
        g = torch.exp(ld.double().clamp(max=0)).view(1, -1, 1, 1)
        check("ds0", got_grad[3], g * p.X, g * p.A, g * p.E, 0, dtype, state=True)


def inputs(T, N, H, dk, dv, dtype, seed, layout="time", odd=0, p_done=0.0, slow=8.0):
    gen = torch.Generator().manual_seed(seed)

    def steps(*widths):
        # "time": [T, N, .], "sequence": stored [N, T, .], all operands side by side in one buffer, `odd` entries behind them
        total = sum(H * w for w in widths) + odd
        t = torch.randn(*((N, T) if layout == "sequence" else (T, N)), total, generator=gen).to(dtype).cuda()
        t = t.transpose(0, 1) if layout == "sequence" else t
        out, at = [], 0
        for w in widths:
            out.append(t[..., at:at + H * w].unflatten(2, (H, w)))
            at += H * w
        return out

    q, k, v = steps(dk, dk, dv)
    do, = steps(dv)
    s0, ds_last = torch.randn(N, H, dk, dv, generator=gen).cuda(), torch.randn(N, H, dk, dv, generator=gen).cuda()
    ld = torch.log1p(-torch.exp2(-torch.linspace(0.5, slow, H, dtype=torch.float64))).float().cuda()
    done = (torch.rand(T, N, generator=gen) < p_done).to(torch.uint8).cuda() if p_done else None
    return q, k, v, ld, s0, done, do, ds_last


CASES = [  # T, N, H, dk, dv: one step, a batch of steps and its edges, a chunk and its edges, several, pieces, ragged widths
    (1, 1, 1, 1, 1), (1, 3, 5, 64, 64), (2, 2, 3, 128, 128), (5, 4, 2, 64, 64), (31, 1, 3, 40, 24), (63, 2, 1, 33, 65), (127, 2, 2, 64, 128),
    (128, 1, 3, 128, 64), (129, 2, 2, 64, 64), (256, 1, 2, 128, 128), (300, 2, 3, 72, 40), (700, 1, 2, 128, 128), (1500, 1, 1, 64, 64),
    (400, 40, 4, 16, 8)]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("layout,odd,p_done", [("time", 0, 0.0), ("sequence", 8, 0.01), ("time", 3, 0.2), ("sequence", 0, 0.0)])
@pytest.mark.parametrize("T,N,H,dk,dv", CASES)
def test_forward_and_backward(T, N, H, dk, dv, layout, odd, p_done, dtype):
    q, k, v, ld, s0, done, do, ds_last = inputs(T, N, H, dk, dv, dtype, T * 1009 + N * 31 + dk + dv, layout, odd, p_done)
    scale = dk ** -0.5
    got = S().linear_attention(q, k, v, ld, s0, done=done)
    grad = S().linear_attention_backward(do, q, k, v, ld, s0, done=done, ds_last=ds_last)
    S().check()
    check_all(q, k, v, ld, s0, done, scale, do, ds_last, got, grad)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("T", [3, 200, 900])
def test_optional_arguments(T, dtype):
    q, k, v, ld, s0, _, do, ds_last = inputs(T, 2, 3, 64, 64, dtype, 1)
    check_all(q, k, v, ld, None, None, 0.3, do, None, S().linear_attention(q, k, v, ld, scale=0.3),
              S().linear_attention_backward(do, q, k, v, ld, scale=0.3))
    check_all(q, k, v, ld, None, None, 0.3, do, ds_last, None, S().linear_attention_backward(do, q, k, v, ld, scale=0.3, ds_last=ds_last))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
def test_steps_one_by_one_are_the_sequence(dtype):
    """Acting with the state kept in place, one step and then some at a time, gives what one call over the rollout gives."""
    q, k, v, ld, s0, done, _, _ = inputs(420, 3, 2, 64, 64, dtype, 3, p_done=0.02)
    state, out, at = s0.clone(), [], 0
    for n in (1, 1, 1, 5, 1, 130, 1, 280):
        o, last = S().linear_attention(q[at:at + n], k[at:at + n], v[at:at + n], ld, state, done=done[at:at + n], s_last=state)
        assert last is state
        out.append(o)
        at += n
    check_all(q, k, v, ld, s0, done, 64 ** -0.5, got=(torch.cat(out), state))


@pytest.mark.parametrize("dtype,T", [(torch.float32, 2000), (torch.bfloat16, 2000), (torch.float16, 1030)])
def test_state_in_place_over_pieces(dtype, T):
    q, k, v, ld, s0, _, _, _ = inputs(T, 1, 2, 64, 64, dtype, 5)
    state = s0.clone()
    o, _ = S().linear_attention(q, k, v, ld, state, s_last=state)
    check_all(q, k, v, ld, s0, None, 0.125, got=(o, state))


@pytest.mark.parametrize("T", [20, 100, 1500])
def test_state_in_place_beside_a_nan(T):
    """One sequence and head meets an infinity: its memory is computed apart from the others', all of them in place."""
    q, k, v, ld, s0, _, _, _ = inputs(T, 2, 2, 64, 64, torch.bfloat16, 15)
    clean, last = S().linear_attention(q, k, v, ld, s0)
    v = v.clone()
    v[T // 2, 1, 0, 9] = float("inf")
    state = s0.clone()
    o, _ = S().linear_attention(q, k, v, ld, state, s_last=state)
    touched = torch.zeros_like(o, dtype=torch.bool)
    touched[T // 2:, 1, 0, 9] = True
    assert not torch.isfinite(o[touched]).any() and not torch.isfinite(state[1, 0, :, 9]).any()
    u = U[torch.bfloat16]
    assert ((o[~touched].double() - clean[~touched].double()).abs() <= 4 * u * (clean[~touched].double().abs() + 8 * float(clean.double().abs().mean()))).all()
    state[1, 0, :, 9] = last[1, 0, :, 9]
    assert ((state - last).abs() <= 1e-4 * (last.abs() + float(last.abs().mean()))).all()


@pytest.mark.parametrize("dk,dv", [(1, 1), (3, 5), (2, 128), (65, 1)])
def test_narrow_heads_on_aligned_rows(dk, dv):
    """Heads of a few entries in 16 bits, in rows padded to 16 bytes: by chunks as well."""
    for dtype in (torch.bfloat16, torch.float16):
        gen = torch.Generator().manual_seed(dk + dv)
        q, k, v, do = (torch.randn(300, 2, 3, (w + 7) // 8 * 8, generator=gen).to(dtype).cuda()[..., :w] for w in (dk, dk, dv, dv))
        s0, ds_last = (torch.randn(2, 3, dk, dv, generator=gen).cuda() for _ in range(2))
        ld = torch.tensor([-0.5, -0.05, -0.01]).cuda()
        o = torch.empty(300, 2, 3, (dv + 7) // 8 * 8, dtype=dtype, device="cuda")[..., :dv]
        got = S().linear_attention(q, k, v, ld, s0, out=o)
        assert got[0] is o
        check_all(q, k, v, ld, s0, None, dk ** -0.5, do, ds_last, got, S().linear_attention_backward(do, q, k, v, ld, s0, ds_last=ds_last))


def test_two_streams_at_once():
    """Calls on two streams side by side, each with a workspace of its own."""
    made = []
    for seed, T in ((31, 1400), (32, 900)):
        made.append((torch.cuda.Stream(), inputs(T, 1, 3, 64, 64, torch.bfloat16, seed, p_done=0.01)))
    torch.cuda.synchronize()
    got = []
    for _ in range(3):
        for stream, (q, k, v, ld, s0, done, do, ds_last) in made:
            with torch.cuda.stream(stream):
                got.append((S().linear_attention(q, k, v, ld, s0, done=done), S().linear_attention_backward(do, q, k, v, ld, s0, done=done, ds_last=ds_last)))
    torch.cuda.synchronize()
    for i, (a, b) in enumerate(got):
        q, k, v, ld, s0, done, do, ds_last = made[i % 2][1]
        check_all(q, k, v, ld, s0, done, 0.125, do, ds_last, a, b)


def test_no_steps_passes_the_state_on():
    e = torch.empty(0, 2, 3, 16, device="cuda")
    s0 = torch.randn(2, 3, 16, 16, device="cuda")
    ld = torch.full((3,), -0.1, device="cuda")
    o, last = S().linear_attention(e, e, e, ld, s0)
    assert o.shape == (0, 2, 3, 16) and torch.equal(last, s0)
    assert torch.equal(S().linear_attention_backward(e, e, e, e, ld, s0, ds_last=s0)[3], s0)
    assert float(S().linear_attention(e, e, e, ld)[1].abs().max()) == 0.0


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("T", [12, 300, 1100])
def test_nothing_passes_a_flag_or_goes_back_in_time(T, dtype):
    """An infinity or a NaN ahead of a flag reaches neither what follows it, nor earlier steps, nor other heads, sequences and
    entries of v."""
    q, k, v, ld, s0, _, do, ds_last = inputs(T, 3, 2, 64, 32, dtype, T)
    done = torch.zeros(T, 3, dtype=torch.bool, device="cuda")
    at = T // 2
    done[at, 0] = done[at, 1] = True
    k, v, q = k.clone(), v.clone(), q.clone()
    clean = S().linear_attention(q, k, v, ld, s0, done=done), S().linear_attention_backward(do, q, k, v, ld, s0, done=done, ds_last=ds_last)
    check_all(q, k, v, ld, s0, done, 0.125, do, ds_last, *clean)
    bad_v, bad_k = v.clone(), k.clone()
    bad_v[at, 0, 1, 5] = float("inf")
    bad_k[at - 3, 1, 0, 7] = float("nan")
    o, last = S().linear_attention(q, bad_k, bad_v, ld, s0, done=done)
    touched = torch.zeros_like(o, dtype=torch.bool)
    touched[at, 0, 1, 5] = True
    touched[at - 3:at + 1, 1, 0] = True
    assert not torch.isfinite(o[touched]).any()
    p = Pass(q, k, v, ld, torch.cat([torch.zeros_like(done[:1]), done[:-1]]), s0, True)
    check("o elsewhere", o[~touched], 0.125 * p.o[~touched], 0.125 * p.a[~touched], 0.125 * p.e[~touched], 64, dtype)
    keep = (~done[-1]).double().view(-1, 1, 1, 1)
    check("last state", last, keep * p.X, keep * p.A, keep * p.E, 0, dtype, state=True)
    # and backwards: a gradient behind the flag does not reach what lies ahead of it
    bad_do = do.clone()
    bad_do[at + 1, 0, 1, 5] = float("inf")
    grad = S().linear_attention_backward(bad_do, q, k, v, ld, s0, done=done, ds_last=ds_last)
    for name, x, y in zip(("dk", "dv"), grad[1:3], clean[1][1:3]):
        same = torch.ones_like(x, dtype=torch.bool)
        same[at + 1, 0, 1] = False
        u = U[dtype]
        assert ((x[same].double() - y[same].double()).abs() <= 8 * u * (y[same].double().abs() + float(y.double().abs().mean()) * 8)).all(), name
        assert torch.isfinite(x[same]).all(), name
    assert not torch.isfinite(grad[0][at + 1, 0, 1]).all() and torch.isfinite(grad[0][:at + 1]).all() and torch.isfinite(grad[0][at + 2:]).all()
    assert torch.isfinite(grad[3]).all()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_extreme_decays(dtype):
    """Heads that forget at once, fade fast, hardly fade, do not fade, and one told to grow (which counts as not fading)."""
    T = 700
    ld = torch.tensor([-float("inf"), -200.0, -3.0, -1e-4, 0.0, 5.0]).cuda()
    q, k, v, _, s0, done, do, ds_last = inputs(T, 2, 6, 32, 32, dtype, 4, p_done=0.005)
    check_all(q, k, v, ld, s0, done, 0.5, do, ds_last, S().linear_attention(q, k, v, ld, s0, done=done, scale=0.5),
              S().linear_attention_backward(do, q, k, v, ld, s0, done=done, scale=0.5, ds_last=ds_last))


@pytest.mark.parametrize("dtype,size", [(torch.float16, 2.0 ** 9), (torch.float16, 2.0 ** -9), (torch.bfloat16, 2.0 ** 40), (torch.bfloat16, 2.0 ** -40)])
def test_large_and_small_values(dtype, size):
    """What is held in between has the range of float32: values whose scores and states leave float16's range."""
    q, k, v, ld, s0, done, do, ds_last = inputs(260, 2, 2, 64, 64, dtype, 6, p_done=0.01)
    k = (k.double() * size).to(dtype)
    q = (q.double() * size).to(dtype)
    s0 = s0 * size
    scale = size ** -2 / 8
    got = S().linear_attention(q, k, v, ld, s0, done=done, scale=scale)
    grad = S().linear_attention_backward(do, q, k, v, ld, s0, done=done, scale=scale, ds_last=ds_last * size)
    check_all(q, k, v, ld, s0, done, scale, do, ds_last * size, got, grad)


def test_broadcast_operands():
    """One key and value for all heads, one query for all sequences: strides of 0."""
    for dtype, T in ((torch.float32, 50), (torch.bfloat16, 260)):
        q, k, v, ld, s0, done, do, ds_last = inputs(T, 3, 4, 64, 64, dtype, 9, p_done=0.02)
        k, v, q = k[:, :, :1].expand(-1, -1, 4, -1), v[:, :, :1].expand(-1, -1, 4, -1), q[:, :1].expand(-1, 3, -1, -1)
        check_all(q, k, v, ld, s0, done, 0.125, do, ds_last, S().linear_attention(q, k, v, ld, s0, done=done),
                  S().linear_attention_backward(do, q, k, v, ld, s0, done=done, ds_last=ds_last))


def test_gradient_of_the_definition():
    """Against torch's derivatives of the definition in 64 bits: within 2e-6 of the largest entry in float32 (some 100 roundings)."""
    q, k, v, ld, s0, done, do, ds_last = inputs(40, 2, 3, 24, 16, torch.float32, 11, p_done=0.1)
    w = [x.double().detach().clone().requires_grad_() for x in (q, k, v, s0)]
    state, total = w[3], 0.0
    for t in range(40):
        state = torch.exp(ld.double()).view(1, 3, 1, 1) * state + w[1][t].unsqueeze(-1) * w[2][t].unsqueeze(-2)
        total = total + (0.4 * (w[0][t].unsqueeze(-1) * state).sum(-2) * do[t].double()).sum()
        state = torch.where(done[t].view(-1, 1, 1, 1) != 0, 0.0, state)
    (total + (state * ds_last.double()).sum()).backward()
    grad = S().linear_attention_backward(do, q, k, v, ld, s0, done=done, scale=0.4, ds_last=ds_last)
    for x, y in zip(grad, w):
        assert float((x.double() - y.grad).abs().max()) <= 2e-6 * float(y.grad.abs().max())


def test_gradient_against_differences():
    """Directional differences of sum(do * o) + sum(ds_last * s_last), from the 32-bit forward pass.  In one operand the value is
    linear, so a difference of any size has no curvature; rounding leaves 1e-5 of the scale, bound 1e-4."""
    q, k, v, ld, s0, done, do, ds_last = inputs(150, 2, 2, 32, 24, torch.float32, 8, p_done=0.05)
    grads = S().linear_attention_backward(do, q, k, v, ld, s0, done=done, ds_last=ds_last)
    gen = torch.Generator().manual_seed(6)

    def value(*a):
        o, last = S().linear_attention(a[0], a[1], a[2], ld, a[3], done=done)
        return float((o.double() * do.double()).sum() + (last.double() * ds_last.double()).sum())

    base = [q, k, v, s0]
    for i, g in enumerate(grads):
        d = torch.randn(g.shape, generator=gen).cuda()
        up, down = (value(*[x + sign * d if j == i else x for j, x in enumerate(base)]) for sign in (1, -1))
        want = float((g.double() * d.double()).sum())
        assert abs((up - down) / 2 - want) <= 1e-4 * float(g.double().norm() * d.double().norm()), i


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_offsets_past_32_bits(dtype):
    """Steps so far apart that the last lie past 2^32 bytes and elements."""
    T, w = 140, 64
    stride = (1 << 32) // 128 + 64
    big = torch.empty(stride * (T - 1) + 3 * w, dtype=dtype, device="cuda")
    gen = torch.Generator().manual_seed(12)
    q, k, v = (big.as_strided((T, 1, 1, w), (stride, w, w, 1), i * w) for i in range(3))
    for x in (q, k, v):
        x.copy_(torch.randn(T, 1, 1, w, generator=gen))
    ld = torch.full((1,), -0.05, device="cuda")
    check_all(q, k, v, ld, None, None, 0.125, got=S().linear_attention(q, k, v, ld))


@pytest.mark.parametrize("T", [1, 300, 1500])
def test_captured_and_replayed(T):
    """Forward and backward in one graph, replayed over changed inputs, beside a graph of its own for other inputs."""
    made = []
    for seed in (21, 22):
        x = inputs(T, 1, 2, 64, 64, torch.bfloat16, seed, p_done=0.01)
        q, k, v, ld, s0, done, do, ds_last = x
        S().linear_attention(q, k, v, ld, s0, done=done)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            got = S().linear_attention(q, k, v, ld, s0, done=done)
            grad = S().linear_attention_backward(do, q, k, v, ld, s0, done=done, ds_last=ds_last)
        made.append((graph, x, got, grad))
    for _, x, _, _ in made:
        x[2].mul_(0.5)
    for graph, *_ in made:
        graph.replay()
    torch.cuda.synchronize()
    for _, (q, k, v, ld, s0, done, do, ds_last), got, grad in made:
        check_all(q, k, v, ld, s0, done, 0.125, do, ds_last, got, grad)
