"""GPU: queries and keys normed by head and turned by position, forward and backward, against 64 bits.

eps = 2^-24, u = half a step of the stored type.  r is off by a sum of dim squares ((dim + 4) / 2 eps) and a reciprocal root (2
eps), a product with it and the weight 2 eps; sine and cosine are off by 2^-22 in all (the angle's fraction of a turn is rounded
to float32, half of it times 2 pi, and the functions to a few units).  So y is within (dim / 2 + 8) eps + 2^-21 of |y_a| + |y_b|,
and then rounded once.  A gradient has one more sum of dim terms, whose terms are taken positive for the bound.
"""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

EPS = 2.0 ** -24
U = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}


def S():
    from paper_1906_04585_b200 import sequence
    return sequence


def turn(x, phase, interleaved):
    n = phase.shape[-1]
    a, b = (x[..., :2 * n:2], x[..., 1:2 * n:2]) if interleaved else (x[..., :n], x[..., n:2 * n])
    c, s = torch.cos(phase), torch.sin(phase)
    a, b = a * c - b * s, b * c + a * s
    t = torch.stack([a, b], -1).flatten(-2) if interleaved else torch.cat([a, b], -1)
    return torch.cat([t, x[..., 2 * n:]], -1)


def spread(x, n, interleaved):
    """|a| + |b| in the place of both, |x| elsewhere."""
    a, b = (x[..., :2 * n:2].abs(), x[..., 1:2 * n:2].abs()) if interleaved else (x[..., :n].abs(), x[..., n:2 * n].abs())
    t = torch.stack([a + b, a + b], -1).flatten(-2) if interleaved else torch.cat([a + b, a + b], -1)
    return torch.cat([t, x[..., 2 * n:].abs()], -1)


def close(name, got, want, err):
    u, tiny = U[got.dtype], 2.0 ** -25 if got.dtype == torch.float16 else 1e-37
    off = (got.double() - want).abs()
    bound = u * want.abs() + tiny + err * (1 + u)
    bad = ~(off <= bound)
    assert not bad.any(), "%s: %d of %d outside, worst %.3g times the bound" % (name, int(bad.sum()), bad.numel(), float((off / bound).max()))


def check(x, w, positions, inv_freq, eps, interleaved, y, dy=None, dx=None, dw=None):
    dim, n = x.shape[-1], inv_freq.shape[0]
    x = x.double()
    wd = torch.ones(dim, dtype=torch.float64, device=x.device) if w is None else w.double()
    phase = (positions.double().unsqueeze(1) * inv_freq.double()).unsqueeze(1)
    r = 1.0 / torch.sqrt(x.pow(2).mean(-1, keepdim=True) + eps)
    if y is not None:
        flat = x * r * wd
        close("y", y, turn(flat, phase, interleaved), ((dim / 2 + 8) * EPS + 2.0 ** -21) * spread(flat, n, interleaved))
    if dy is None:
        return
    e = turn(dy.double(), -phase, interleaved)
    ee = spread(dy.double(), n, interleaved)            # e's own error is 2^-21 of this
    xh = x * r
    dot = (e * wd * xh).mean(-1, keepdim=True)
    dots = (ee * wd.abs() * xh.abs()).mean(-1, keepdim=True)
    want = r * (e * wd - xh * dot)
    close("dx", dx, want, r * (2.0 ** -21 + (2 * dim + 16) * EPS) * (ee * wd.abs() + xh.abs() * dots))
    rows = xh.shape[0] * xh.shape[1]
    sums = (e * xh).sum((0, 1))
    # a sum of `rows` terms by a tree of lanes, blocks and warps no deeper than rows / 64 + 64
    close("dw", dw, sums, (2.0 ** -21 + (dim / 2 + 16 + rows / 64 + 64) * EPS) * (ee * xh.abs()).sum((0, 1)))


def inputs(n, hq, hk, dim, pairs, dtype, wdtype, seed, layout, far=5000):
    gen = torch.Generator().manual_seed(seed)
    odd = {"flat": 0, "slices": 2 * hk * dim, "odd": 3, "heads": 0}[layout]
    if layout == "heads":       # head before token
        q, k = (torch.randn(h, n, dim, generator=gen).to(dtype).cuda().transpose(0, 1) for h in (hq, hk))
    else:
        both = torch.randn(n, (hq + hk) * dim + odd, generator=gen).mul_(1.5).to(dtype).cuda()
        q, k = both[:, :hq * dim].unflatten(1, (hq, dim)), both[:, hq * dim:(hq + hk) * dim].unflatten(1, (hk, dim))
    wq, wk = ((torch.randn(dim, generator=gen) * 0.2 + 1).to(wdtype).cuda() for _ in range(2))
    positions = torch.randint(-far, far, (n,), generator=gen).to(torch.int32).cuda()
    inv_freq = torch.pow(10000.0, -torch.arange(pairs, dtype=torch.float64) / max(1, pairs)).float().cuda()
    dq, dk = torch.randn(n, hq, dim, generator=gen).to(dtype).cuda(), torch.randn(n, hk, dim, generator=gen).to(dtype).cuda()
    return q, k, wq, wk, positions, inv_freq, dq, dk


CASES = [  # n, hq, hk, dim, pairs
    (1, 1, 1, 1, 0), (1, 8, 8, 64, 32), (3, 5, 2, 128, 64), (7, 2, 1, 2, 1), (33, 4, 4, 75, 20), (50, 3, 1, 80, 40), (64, 16, 2, 256, 128),
    (100, 1, 3, 96, 16), (19, 6, 2, 64, 30), (9, 2, 2, 255, 127), (5000, 2, 1, 64, 32), (700, 40, 0, 40, 20), (5, 0, 3, 32, 0)]


@pytest.mark.parametrize("dtype,wdtype", [(torch.float32, torch.float32), (torch.bfloat16, torch.bfloat16), (torch.bfloat16, torch.float32),
                                          (torch.float16, torch.float16)])
@pytest.mark.parametrize("layout", ["flat", "slices", "odd", "heads"])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("n,hq,hk,dim,pairs", CASES)
def test_forward_and_backward(n, hq, hk, dim, pairs, interleaved, layout, dtype, wdtype):
    q, k, wq, wk, positions, inv_freq, dq, dk = inputs(n, hq, hk, dim, pairs, dtype, wdtype, n + dim, layout)
    yq, yk = S().qk_norm_rotary(q, k, positions, inv_freq, wq, wk, interleaved=interleaved)
    g = S().qk_norm_rotary_backward(dq, dk, q, k, positions, inv_freq, wq, wk, interleaved=interleaved)
    check(q, wq, positions, inv_freq, 1e-6, interleaved, yq, dq, g[0], g[2])
    check(k, wk, positions, inv_freq, 1e-6, interleaved, yk, dk, g[1], g[3])


def test_far_positions():
    """At position 2^31 - 1 the first pair has turned 2^31 radians: the angle is formed in 64 bits."""
    q, k, wq, wk, _, inv_freq, dq, dk = inputs(64, 2, 2, 128, 64, torch.float32, torch.float32, 5, "flat")
    positions = (torch.arange(64, device="cuda") * 34087042).to(torch.int32)
    positions[-1], positions[0] = 2 ** 31 - 1, -2 ** 31
    yq, yk = S().qk_norm_rotary(q, k, positions, inv_freq, wq, wk)
    check(q, wq, positions, inv_freq, 1e-6, False, yq)


def test_in_place_and_without_weights():
    for interleaved in (False, True):
        q, k, _, _, positions, inv_freq, dq, dk = inputs(100, 4, 2, 64, 32, torch.bfloat16, torch.float32, 3, "slices")
        q0, k0 = q.clone(), k.clone()
        yq, yk = S().qk_norm_rotary(q, k, positions, inv_freq, interleaved=interleaved, q_out=q, k_out=k)
        assert yq is q and yk is k
        check(q0, None, positions, inv_freq, 1e-6, interleaved, q)
        check(k0, None, positions, inv_freq, 1e-6, interleaved, k)
        dq0, dk0 = dq.clone(), dk.clone()
        g = S().qk_norm_rotary_backward(dq, dk, q0, k0, positions, inv_freq, interleaved=interleaved, dq=dq, dk=dk)
        check(q0, None, positions, inv_freq, 1e-6, interleaved, None, dq0, dq, g[2])
        check(k0, None, positions, inv_freq, 1e-6, interleaved, None, dk0, dk, g[3])


def test_rows_without_anything_and_beyond():
    """A head of zeros stays zero; a NaN or an infinity stays in its head, and in its entry of the weights' gradients."""
    q, k, wq, wk, positions, inv_freq, dq, dk = inputs(40, 3, 1, 64, 32, torch.float32, torch.float32, 8, "flat")
    q = q.clone()
    q[3, 1] = 0.0
    y, _ = S().qk_norm_rotary(q, k, positions, inv_freq, wq, wk)
    assert float(y[3, 1].abs().max()) == 0.0
    want = y.clone()
    q[5, 2, 7] = float("nan")
    y, _ = S().qk_norm_rotary(q, k, positions, inv_freq, wq, wk)
    assert torch.isnan(y[5, 2]).all()
    y[5, 2] = want[5, 2]
    assert torch.equal(y, want)


def test_same_bits_every_time():
    q, k, wq, wk, positions, inv_freq, dq, dk = inputs(3000, 6, 2, 128, 64, torch.bfloat16, torch.float32, 4, "slices")
    first = S().qk_norm_rotary_backward(dq, dk, q, k, positions, inv_freq, wq, wk)
    for _ in range(3):
        assert all(torch.equal(a, b) for a, b in zip(first, S().qk_norm_rotary_backward(dq, dk, q, k, positions, inv_freq, wq, wk)))


def test_no_tokens():
    e = torch.empty(0, 2, 64, device="cuda")
    positions, inv_freq = torch.empty(0, dtype=torch.int32, device="cuda"), torch.ones(32, device="cuda")
    assert S().qk_norm_rotary(e, e, positions, inv_freq)[0].shape == (0, 2, 64)
    g = S().qk_norm_rotary_backward(e, e, e, e, positions, inv_freq)
    assert float(g[2].abs().max()) == 0.0 and float(g[3].abs().max()) == 0.0


def test_gradient_against_differences():
    """Directional differences of sum(dq * q_out) + sum(dk * k_out) with h = 1/64 from the 32-bit forward pass: curvature leaves
    h^2 / 6 of a third derivative no larger than some ten times the slope's scale (4e-4), rounding 1e-5; bound 2e-3."""
    q, k, wq, wk, positions, inv_freq, dq, dk = inputs(60, 3, 2, 48, 20, torch.float32, torch.float32, 7, "flat")
    grads = S().qk_norm_rotary_backward(dq, dk, q, k, positions, inv_freq, wq, wk)
    gen = torch.Generator().manual_seed(2)

    def value(*a):
        y, z = S().qk_norm_rotary(a[0], a[1], positions, inv_freq, a[2], a[3])
        return float((y.double() * dq.double()).sum() + (z.double() * dk.double()).sum())

    base = [q, k, wq, wk]
    for i, g in enumerate(grads):
        d = torch.randn(g.shape, generator=gen).cuda() / 64
        up, down = (value(*[x + sign * d if j == i else x for j, x in enumerate(base)]) for sign in (1, -1))
        want = float((g.double() * d.double()).sum())
        assert abs((up - down) / 2 - want) <= 2e-3 * float(g.double().norm() * d.double().norm()), i


def test_offsets_past_32_bits():
    n, dim = 40, 64
    stride = (1 << 32) // 32 + 64
    big = torch.empty(stride * (n - 1) + 2 * dim, dtype=torch.bfloat16, device="cuda")
    gen = torch.Generator().manual_seed(12)
    q, k = (big.as_strided((n, 1, dim), (stride, dim, 1), i * dim) for i in range(2))
    for x in (q, k):
        x.copy_(torch.randn(n, 1, dim, generator=gen))
    positions = torch.arange(n, dtype=torch.int32, device="cuda")
    inv_freq = torch.linspace(1, 0.01, 32, device="cuda")
    yq, yk = S().qk_norm_rotary(q, k, positions, inv_freq)
    check(q, None, positions, inv_freq, 1e-6, False, yq)
    check(k, None, positions, inv_freq, 1e-6, False, yk)
