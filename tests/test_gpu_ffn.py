"""GPU: the gated feed-forward block, forward and backward, against the formulas in 64 bits.

Bounds.  u = 2^-8 (bfloat16) or 2^-11 (float16, plus half its smallest step, 2^-25) is the rounding of a stored value.
A tensor-core sum of n exact products is within n 2^-24 of the sum of their magnitudes (no rounding is assumed to be
better than truncation, hence 2 n 2^-24 below); the activations' fast exponential and division add 2^-20 of a value.  p, g, u, dg
and du are rounded once each before they are operands, so with P(z) an upper bound on the error of z and |.| the
elementwise magnitude:
  P(g) = k |x||Wg|^T                   stored: + u |g|
  P(p) = |act g| P(u) + lip |u| P(g) + 2^-20 |p| + u |p|,   P(y) = P(p) |Wd|^T + k |p||Wd|^T + u |y|
with lip = 1.13, the largest slope of the three activations; the second derivative is at most 0.8 away from relu's kink.
Gradients use the stored g and u:
  P(dp) = k |dy||Wd|    P(dg) = |u s| P(dp) + |dp| (|s| P'(u) + 0.8 |u| P'(g)) + 2^-19 |dg| + u |dg|
and the same for du, dx and the weight gradients.  relu's slope jumps at 0: elements whose g is within its own error of 0
are exempt there (and what they move is covered by adding their whole contribution to the bound)."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

EPS = 2.0 ** -24
U = {torch.bfloat16: (2.0 ** -8, 0.0), torch.float16: (2.0 ** -11, 2.0 ** -25)}
LIP = 1.13


def S():
    from paper_1906_04585_b200 import sequence
    return sequence


def act(g, kind):
    if kind == "silu":
        s = torch.sigmoid(g)
        return g * s, s * (1 + g * (1 - s))
    if kind == "gelu":
        phi = 0.5 * torch.special.erfc(-g / 2 ** 0.5)
        return g * phi, phi + g * torch.exp(-g * g / 2) / (2 * torch.pi) ** 0.5
    return torch.clamp(g, min=0), (g > 0).double()


def check(name, got, want, err):
    u, tiny = U[got.dtype]
    off = (got.double() - want).abs()
    bound = (err + u * want.abs()) * (1 + u) + tiny
    bad = ~(off <= bound)
    assert not bad.any(), "%s: %d of %d outside, worst %.3g times the bound" % (name, int(bad.sum()), bad.numel(), float((off / bound).max()))


def make(M, D, F, dtype, seed, pad=0):
    gen = torch.Generator().manual_seed(seed)

    def mat(n, m, std):
        ld = (m + 7) // 8 * 8 + pad
        return (torch.randn(n, ld, generator=gen) * std).to(dtype).cuda()[:, :m]

    return (mat(M, D, 1.0), mat(F, D, D ** -0.5), mat(F, D, D ** -0.5), mat(D, F, F ** -0.5), mat(M, D, 1.0))


def reference(x, wg, wu, wd, dy, kind):
    u, tiny = U[x.dtype]
    x, wg, wu, wd, dy = (t.double() for t in (x, wg, wu, wd, dy))
    M, D = x.shape
    F = wg.shape[0]
    kD, kF, kM = 2 * (D + 64) * EPS, 2 * (F + 64) * EPS, 2 * (M + 64) * EPS
    g, up = x @ wg.T, x @ wu.T
    eg, eu = kD * (x.abs() @ wg.abs().T), kD * (x.abs() @ wu.abs().T)
    v, s = act(g, kind)
    p = v * up
    ep = v.abs() * eu + LIP * eg * (up.abs() + eu) + 2.0 ** -20 * p.abs()
    ep = ep + u * (p.abs() + ep) + tiny
    y = p @ wd.T
    out = {"y": (y, ep @ wd.abs().T + kF * (p.abs() @ wd.abs().T))}
    # stored pre-activations
    eg, eu = eg + u * (g.abs() + eg) + tiny, eu + u * (up.abs() + eu) + tiny
    dp = dy @ wd
    edp = kD * (dy.abs() @ wd.abs())
    kink = (g.abs() <= eg).double() if kind == "relu" else torch.zeros_like(g)
    es = 0.8 * eg + kink
    dg, du = dp * up * s, dp * v
    edg = (up.abs() + eu) * (s.abs() + es) * edp + dp.abs() * (s.abs() * eu + es * (up.abs() + eu)) + 2.0 ** -19 * (dg.abs() + dp.abs() * up.abs() * 0.1)
    edu = (v.abs() + LIP * eg) * edp + dp.abs() * LIP * eg + 2.0 ** -19 * du.abs()
    edg, edu = edg + u * (dg.abs() + edg) + tiny, edu + u * (du.abs() + edu) + tiny
    out["dx"] = (dg @ wg + du @ wu, edg @ wg.abs() + edu @ wu.abs() + 2 * kF * (dg.abs() @ wg.abs() + du.abs() @ wu.abs()))
    out["dw_gate"] = (dg.T @ x, edg.T @ x.abs() + kM * (dg.abs().T @ x.abs()))
    out["dw_up"] = (du.T @ x, edu.T @ x.abs() + kM * (du.abs().T @ x.abs()))
    out["dw_down"] = (dy.T @ p, dy.abs().T @ ep + kM * (dy.abs().T @ p.abs()))
    return out


SHAPES = [  # rows, dim, hidden: one row; each width of the few-rows kernel and one past it; ragged everything; several tiles
    (1, 8, 8), (1, 512, 1024), (7, 2048, 640), (16, 100, 72), (17, 264, 200), (32, 64, 64), (33, 129, 65), (64, 1024, 2048), (65, 328, 520),
    (128, 512, 384), (129, 512, 384), (255, 72, 1000), (256, 256, 128), (300, 1001, 333), (513, 640, 1288), (1024, 512, 2048), (2500, 264, 648)]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("M,D,F", SHAPES)
@pytest.mark.parametrize("kind,pad", [("silu", 0), ("gelu", 8), ("relu", 24)])
def test_forward_and_backward(M, D, F, kind, pad, dtype):
    x, wg, wu, wd, dy = make(M, D, F, dtype, M + 7 * D + 13 * F, pad)
    want = reference(x, wg, wu, wd, dy, kind)
    y, _ = S().gated_ffn(x, wg, wu, wd, kind)
    check("y", y, *want["y"])
    y2, saved = S().gated_ffn(x, wg, wu, wd, kind, save=True)
    assert torch.equal(y, y2)
    grads = S().gated_ffn_backward(dy, x, wg, wu, wd, saved, kind)
    for name, got in zip(("dx", "dw_gate", "dw_up", "dw_down"), grads):
        check(name, got, *want[name])
    again = S().gated_ffn_backward(dy, x, wg, wu, wd, saved, kind)      # saved is not consumed, and the same bits come out
    for p, q in zip(grads, again):
        assert torch.equal(p, q)
    S().check()


def test_outputs_in_place_of_new_tensors_and_untouched_padding():
    M, D, F = 200, 104, 96
    x, wg, wu, wd, dy = make(M, D, F, torch.bfloat16, 1)
    wide = torch.full((M, D + 24), 7.0, dtype=torch.bfloat16, device="cuda")
    y, saved = S().gated_ffn(x, wg, wu, wd, out=wide[:, 8:8 + D], save=True)
    assert float((wide[:, :8] - 7).abs().max()) == 0 and float((wide[:, 8 + D:] - 7).abs().max()) == 0
    assert torch.equal(y, S().gated_ffn(x, wg, wu, wd)[0])
    big = torch.full((F, D + 8), 7.0, dtype=torch.bfloat16, device="cuda")
    got = S().gated_ffn_backward(dy, x, wg, wu, wd, saved, dw_up=big[:, :D])
    assert torch.equal(got[2], S().gated_ffn_backward(dy, x, wg, wu, wd, saved)[2])
    assert float((big[:, D:] - 7).abs().max()) == 0


def test_no_rows():
    x, wg, wu, wd, dy = make(0, 64, 96, torch.bfloat16, 2)
    y, saved = S().gated_ffn(x, wg, wu, wd, save=True)
    assert y.shape == (0, 64)
    grads = S().gated_ffn_backward(dy, x, wg, wu, wd, saved)
    for g in grads[1:]:
        assert float(g.float().abs().sum()) == 0.0


@pytest.mark.parametrize("M", [5, 300])
def test_bad_rows_stay_apart(M):
    x, wg, wu, wd, dy = make(M, 256, 320, torch.bfloat16, 3)
    clean, _ = S().gated_ffn(x, wg, wu, wd)
    x[2, 5] = float("inf")
    x[4, 0] = float("nan")
    y, _ = S().gated_ffn(x, wg, wu, wd)
    keep = [i for i in range(M) if i not in (2, 4)]
    assert torch.equal(y[keep], clean[keep])
    assert torch.isnan(y[4]).all()


def test_large_pre_activations():
    """Gates far outside the exponential's range: silu(-g) is 0 and silu(g) is g, never NaN."""
    for M in (3, 140):
        x = torch.full((M, 64), 100.0, dtype=torch.bfloat16, device="cuda")
        wg = torch.ones(64, 64, dtype=torch.bfloat16, device="cuda")
        wg[::2] = -1
        wu = torch.full((64, 64), 0.01, dtype=torch.bfloat16, device="cuda")
        wd = torch.eye(64, dtype=torch.bfloat16, device="cuda")
        dy = torch.ones(M, 64, dtype=torch.bfloat16, device="cuda")
        for kind in ("silu", "gelu", "relu"):
            y, saved = S().gated_ffn(x, wg, wu, wd, kind, save=True)
            assert torch.isfinite(y).all() and float(y[:, ::2].float().abs().max()) == 0.0
            assert float((y[:, 1::2].double() / (6400.0 * 6400.0 * float(wu[0, 0])) - 1).abs().max()) < 2 ** -6
            for g in S().gated_ffn_backward(dy, x, wg, wu, wd, saved, kind):
                assert torch.isfinite(g).all()


def test_gradient_against_differences():
    """Directional differences of sum(dy * y) from the forward pass.  float16, weights moved by 1/8 of their scale along
    a random direction: curvature leaves below 2 % of the scale of the derivative, float16 rounding of p and y
    (2^-11 each over 128 x 96 independent elements, against a difference of 1/8) below 1 %; bound 5 %."""
    M, D, F = 128, 96, 192
    x, wg, wu, wd, dy = make(M, D, F, torch.float16, 4)
    _, saved = S().gated_ffn(x, wg, wu, wd, save=True)
    grads = S().gated_ffn_backward(dy, x, wg, wu, wd, saved)
    gen = torch.Generator().manual_seed(5)
    args = [x, wg, wu, wd]
    for i, g in enumerate(grads):
        v = (torch.sign(g.float()) * torch.rand(g.shape, generator=gen).cuda() * args[i].float().std() / 8).to(torch.float16)
        up, down = [list(args), list(args)]
        up[i], down[i] = args[i] + v, args[i] - v
        moved = (up[i].double() - down[i].double())
        slope = float(((S().gated_ffn(*up)[0].double() - S().gated_ffn(*down)[0].double()) * dy.double()).sum())
        want = float((g.double() * moved).sum())
        assert abs(slope - want) <= 0.05 * abs(want), (i, slope, want)


def test_other_stream_and_graph():
    x, wg, wu, wd, dy = make(300, 256, 384, torch.bfloat16, 6)
    want = S().gated_ffn(x, wg, wu, wd)[0]
    few = S().gated_ffn(x[:9], wg, wu, wd)[0]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    out = torch.empty_like(want)
    with torch.cuda.stream(side):
        assert torch.equal(S().gated_ffn(x, wg, wu, wd)[0], want)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            S().gated_ffn(x, wg, wu, wd, out=out)
            out[:9] = S().gated_ffn(x[:9], wg, wu, wd)[0]
    out.zero_()
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(out[9:], want[9:]) and torch.equal(out[:9], few)
