"""GPU: the gated linear recurrence, forward and backward, against a step-by-step evaluation in 64 bits.

Bounds come from a running error analysis beside the 64-bit evaluation.  eps = 2^-24.  The smaller of the two gate
weights is within (4 + 2 |f|) eps of itself (fast exponential and division), a step adds that times |x - c| and two
roundings of the result, and passes the earlier error on scaled by a; the maps that join pieces of the time axis pass
through the same sums up to three more times, hence the factor 4 over the analysis of one sequential pass.  Then one
rounding to the stored type.
"""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

EPS = 2.0 ** -24
U = {torch.float32: (2.0 ** -24, 0.0), torch.bfloat16: (2.0 ** -8, 0.0), torch.float16: (2.0 ** -11, 2.0 ** -25)}


def S():
    from paper_1906_04585_b200 import sequence
    return sequence


def check(name, got, want, err):
    u, tiny = U[got.dtype]
    off = (got.double() - want).abs()
    bound = u * want.abs() + tiny + 4 * err * (1 + u) + 1e-38
    bad = ~(off <= bound)
    assert not bad.any(), "%s: %d of %d outside, worst %.3g times the bound" % (name, int(bad.sum()), bad.numel(), float((off / bound).max()))


def reference(f, x, h0, done, dh=None, dh_last=None):
    """dict of (value, error of a sequential 32-bit evaluation) in 64 bits, step by step."""
    T, N, D = x.shape
    f, x = f.double(), x.double()
    a, b = torch.sigmoid(f), torch.sigmoid(-f)
    small = torch.minimum(a, b)
    rel = (4 + 2 * f.abs()) * EPS
    c = torch.zeros(N, D, dtype=torch.float64, device=x.device) if h0 is None else h0.double()
    ec = torch.zeros_like(c)
    h, eh, before, ebefore = (torch.zeros(T, N, D, dtype=torch.float64, device=x.device) for _ in range(4))
    cut = None if done is None else (done != 0)
    for t in range(T):
        before[t], ebefore[t] = c, ec
        h[t] = a[t] * c + b[t] * x[t]
        eh[t] = a[t] * ec + rel[t] * small[t] * (x[t] - c).abs() + 2 * EPS * (h[t].abs() + small[t] * (x[t] - c).abs())
        c, ec = h[t], eh[t]
        if cut is not None:
            c, ec = torch.where(cut[t][:, None], 0.0, c), torch.where(cut[t][:, None], 0.0, ec)
    out = {"h": (h, eh), "h_last": (c, ec)}
    if dh is None and dh_last is None:
        return out
    q = torch.zeros(N, D, dtype=torch.float64, device=x.device) if dh_last is None else dh_last.double()
    eq = torch.zeros_like(q)
    df, edf, dx, edx = (torch.zeros(T, N, D, dtype=torch.float64, device=x.device) for _ in range(4))
    for t in range(T - 1, -1, -1):
        if cut is not None:
            q, eq = torch.where(cut[t][:, None], 0.0, q), torch.where(cut[t][:, None], 0.0, eq)
        own = torch.zeros_like(q) if dh is None else dh[t].double()
        g = own + q
        eg = eq + EPS * g.abs()
        diff = before[t] - x[t]
        dx[t], edx[t] = b[t] * g, b[t] * eg + (rel[t] + 2 * EPS) * b[t] * g.abs()
        df[t] = g * diff * a[t] * b[t]
        edf[t] = a[t] * b[t] * (eg * diff.abs() + g.abs() * (ebefore[t] + EPS * diff.abs())) + (2 * rel[t] + 5 * EPS) * df[t].abs()
        q, eq = a[t] * g, a[t] * eg + (rel[t] + 2 * EPS) * a[t] * g.abs()
    out.update(df=(df, edf), dx=(dx, edx), dh0=(q, eq))
    return out


def inputs(T, N, D, dtype, seed, layout, odd, p_done):
    gen = torch.Generator().manual_seed(seed)

    def steps(std=1.0, mean=0.0):
        # layout "time": [T, N, D]; "sequence": stored [N, T, D]; "half": half of a wider projection
        extra = {"half": D + odd, "time": odd, "sequence": odd}[layout]
        shape = (N, T, D + extra) if layout == "sequence" else (T, N, D + extra)
        t = (torch.randn(*shape, generator=gen) * std + mean).to(dtype).cuda()[..., :D]
        return t.transpose(0, 1) if layout == "sequence" else t

    f, x, dh = steps(2.0, 1.0), steps(), steps()
    h0, dh_last = torch.randn(N, D, generator=gen).cuda(), torch.randn(N, D, generator=gen).cuda()
    done = (torch.rand(T, N, generator=gen) < p_done).to(torch.uint8).cuda() if p_done else None
    return f, x, h0, done, dh, dh_last


CASES = [  # T, N, D: one piece, its edges, a block, a cluster, several turns of a cluster, many sequences, ragged channels
    (1, 1, 1), (1, 5, 96), (2, 3, 33), (15, 2, 64), (16, 2, 64), (17, 2, 70), (31, 1, 128), (100, 3, 5), (128, 2, 64), (129, 1, 66),
    (257, 2, 31), (1024, 1, 64), (1025, 1, 40), (2500, 2, 72), (33, 40, 130), (5, 300, 34)]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("layout,odd,p_done", [("time", 0, 0.0), ("half", 0, 0.1), ("sequence", 2, 0.01), ("time", 1, 0.3)])
@pytest.mark.parametrize("T,N,D", CASES)
def test_forward_and_backward(T, N, D, layout, odd, p_done, dtype):
    f, x, h0, done, dh, dh_last = inputs(T, N, D, dtype, T * 1009 + N * 31 + D, layout, odd, p_done)
    want = reference(f, x, h0, done, dh, dh_last)
    h, last, states = S().gated_recurrence(f, x, h0, done=done, save=True)
    check("h", h, *want["h"])
    check("h_last", last, *want["h_last"])
    df, dx, dh0 = S().gated_recurrence_backward(dh, f, x, states, done=done, dh_last=dh_last)
    check("df", df, *want["df"])
    check("dx", dx, *want["dx"])
    check("dh0", dh0, *want["dh0"])
    assert torch.equal(h, S().gated_recurrence(f, x, h0, done=done)[0])      # with or without stored states: the same bits


def test_optional_arguments():
    f, x, h0, done, dh, dh_last = inputs(70, 2, 48, torch.float32, 1, "time", 0, 0.0)
    h, last, states = S().gated_recurrence(f, x, save=True)
    want = reference(f, x, None, None, dh)
    check("h", h, *want["h"])
    df, dx, dh0 = S().gated_recurrence_backward(dh, f, x, states)
    check("df", df, *want["df"])
    want = reference(f, x, None, None, None, dh_last)
    df, dx, dh0 = S().gated_recurrence_backward(None, f, x, states, dh_last=dh_last)
    check("dx of the last state alone", dx, *want["dx"])
    check("dh0 of the last state alone", dh0, *want["dh0"])


def test_steps_one_by_one_are_the_sequence():
    """Acting with the state kept in place gives what one call over the rollout gives."""
    f, x, h0, done, _, _ = inputs(40, 6, 64, torch.float32, 3, "time", 0, 0.2)
    want = reference(f, x, h0, done)
    state = h0.clone()
    out = []
    for t in range(40):
        h, _, _ = S().gated_recurrence(f[t:t + 1], x[t:t + 1], state, done=done[t:t + 1], h_last=state)
        out.append(h)
    check("h", torch.cat(out), *want["h"])
    check("state", state, *want["h_last"])


def test_no_steps_passes_the_state_on():
    e = torch.empty(0, 3, 20, device="cuda")
    h0 = torch.randn(3, 20, device="cuda")
    h, last, states = S().gated_recurrence(e, e, h0, save=True)
    assert h.shape == (0, 3, 20) and torch.equal(last, h0)
    _, _, dh0 = S().gated_recurrence_backward(e, e, e, states, dh_last=h0)
    assert torch.equal(dh0, h0)
    last = S().gated_recurrence(e, e)[1]
    assert float(last.abs().max()) == 0.0


@pytest.mark.parametrize("T", [12, 90, 1500])
def test_nothing_passes_a_flag(T):
    """An infinity or a NaN ahead of a flag does not reach what follows it, nor the other channels and sequences."""
    f, x, h0, _, dh, dh_last = inputs(T, 3, 34, torch.float32, T, "time", 0, 0.0)
    done = torch.zeros(T, 3, dtype=torch.bool, device="cuda")
    at = T // 2
    done[at, 0] = done[at, 1] = True
    clean = reference(f, x, h0, done, dh, dh_last)
    x = x.clone()
    x[at, 0, 5] = float("inf")
    x[at - 3, 1, 7] = float("nan")
    h, last, states = S().gated_recurrence(f, x, h0, done=done, save=True)
    touched = torch.zeros(T, 3, 34, dtype=torch.bool, device="cuda")
    touched[at, 0, 5] = True
    touched[at - 3:at + 1, 1, 7] = True
    assert not torch.isfinite(h[touched]).any()
    check("h elsewhere", h[~touched], clean["h"][0][~touched], clean["h"][1][~touched])
    check("last state", last, *clean["h_last"])
    # and backwards: a gradient behind the flag does not reach what lies ahead of it
    x = inputs(T, 3, 34, torch.float32, T, "time", 0, 0.0)[1]
    _, _, states = S().gated_recurrence(f, x, h0, done=done, save=True)
    dh = dh.clone()
    dh[at + 1, 0, 5] = float("inf")
    df, dx, dh0 = S().gated_recurrence_backward(dh, f, x, states, done=done, dh_last=dh_last)
    touched[:] = False
    touched[at + 1, 0, 5] = True
    check("dx elsewhere", dx[~touched], clean["dx"][0][~touched], clean["dx"][1][~touched])
    check("dh0", dh0, *clean["dh0"])


def test_extreme_gates():
    """Gates that are all but shut or open keep their digits; a wiped memory leaves nothing behind."""
    T = 300
    gen = torch.Generator().manual_seed(4)
    f = torch.tensor([-200.0, -60.0, -12.0, 0.0, 12.0, 60.0, 200.0, 9.0]).repeat(8).cuda().expand(T, 1, 64).contiguous()
    f[150] = -60.0
    x = torch.randn(T, 1, 64, generator=gen).cuda()
    x[100] *= 1e6
    h0 = torch.randn(1, 64, generator=gen).cuda() * 1e4
    dh = torch.randn(T, 1, 64, generator=gen).cuda()
    want = reference(f, x, h0, None, dh)
    h, last, states = S().gated_recurrence(f, x, h0, save=True)
    check("h", h, *want["h"])
    df, dx, dh0 = S().gated_recurrence_backward(dh, f, x, states)
    check("df", df, *want["df"])
    check("dx", dx, *want["dx"])


def test_gradient_against_differences():
    """Directional differences of sum(dh * h) + sum(dh_last * h_last) in 64 bits from the 32-bit forward pass, h = 1/64:
    curvature leaves below 2.4e-4 of the scale, rounding 2 eps / h = 8e-6; bound 1e-3."""
    f, x, h0, done, dh, dh_last = inputs(150, 2, 34, torch.float32, 8, "time", 0, 0.05)
    _, _, states = S().gated_recurrence(f, x, h0, done=done, save=True)
    df, dx, dh0 = S().gated_recurrence_backward(dh, f, x, states, done=done, dh_last=dh_last)
    gen = torch.Generator().manual_seed(6)

    def value(f_, x_, h0_):
        h, last, _ = S().gated_recurrence(f_, x_, h0_, done=done)
        return float((h.double() * dh.double()).sum() + (last.double() * dh_last.double()).sum())

    for name, grad, args in (("f", df, lambda v: (f + v, x, h0)), ("x", dx, lambda v: (f, x + v, h0)), ("h0", dh0, lambda v: (f, x, h0 + v))):
        v = torch.randn(grad.shape, generator=gen).cuda() / 64
        slope = (value(*args(v)) - value(*args(-v))) / 2
        want = float((grad.double() * v.double()).sum())
        scale = float(grad.double().norm() * v.double().norm())
        assert abs(slope - want) <= 1e-3 * scale, (name, slope, want, scale)


def test_offsets_past_32_bits():
    """2^32 elements of f and x apart in time: a strided view of one large buffer."""
    D, T = 64, 40
    stride = (1 << 32) // 32 + 64            # 33 steps span more than 2^32 elements
    big = torch.empty(stride * (T - 1) + 2 * D, dtype=torch.bfloat16, device="cuda")
    f = big.as_strided((T, 1, D), (stride, 2 * D, 1))
    x = big.as_strided((T, 1, D), (stride, 2 * D, 1), D)
    gen = torch.Generator().manual_seed(12)
    f.copy_(torch.randn(T, 1, D, generator=gen))
    x.copy_(torch.randn(T, 1, D, generator=gen))
    want = reference(f, x, None, None)
    h, _, _ = S().gated_recurrence(f, x)
    check("h", h, *want["h"])
