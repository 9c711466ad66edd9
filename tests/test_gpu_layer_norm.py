"""GPU: layer norm forward and backward against the formulas in 64 bits.

Bounds.  u = 2^-24 / 2^-8 / 2^-11 is half a unit in the last place of the stored type (float16 adds 2^-25, half its
smallest step), eps = 2^-24.  A row of up to 16384 elements is added in at most 16 + 10 levels, so its mean is within
27 eps of mean |s|, its variance within 32 eps (+ the mean's error squared), rstd within 20 eps; with the subtraction,
the two products and the bias y is within 64 eps of |xh w| + mean|s| rstd |w| + |b|, and rounded once.  The backward
pass starts from those statistics and adds two more such sums: 128 eps of what it adds up.  A column sum over the rows
adds at most rows / 4 numbers in one chain here, and 64 more in the joins.
"""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

EPS = 2.0 ** -24
U = {torch.float32: (2.0 ** -24, 0.0), torch.bfloat16: (2.0 ** -8, 0.0), torch.float16: (2.0 ** -11, 2.0 ** -25)}


def S():
    from paper_1906_04585_b200 import sequence
    return sequence


def check(name, got, want, scale, k, extra=0.0):
    """|got - want| <= u |want| + k eps scale, element by element."""
    u, tiny = U[got.dtype]
    off = (got.double() - want).abs()
    bound = u * want.abs() + tiny + k * EPS * scale * (1 + u) + extra
    bad = ~(off <= bound)
    assert not bad.any(), "%s: %d of %d outside, worst %.3g times the bound" % (name, int(bad.sum()), bad.numel(), float((off / bound).max()))


def rows_of(rows, cols, pad, dtype, gen, std=1.0, mean=0.0):
    wide = (torch.randn(rows, cols + pad, generator=gen, dtype=torch.float64) * std + mean).to(dtype).cuda()
    return wide[:, :cols]


def reference(x, res, w, b, eps):
    s = x.double() if res is None else x.double() + res.double()
    mean = s.mean(1, keepdim=True)
    var = ((s - mean) ** 2).mean(1, keepdim=True)
    rstd = 1.0 / torch.sqrt(var + eps)
    xh = (s - mean) * rstd
    wd = torch.ones_like(xh[:1]) if w is None else w.double()
    bd = torch.zeros_like(xh[:1]) if b is None else b.double()
    return s, mean, rstd, xh, xh * wd + bd, wd, bd


SHAPES = [(1, 1), (3, 7), (5, 32), (2, 255), (33, 512), (130, 513), (9, 1000), (700, 2048), (3, 4104), (3, 5000), (2, 8200), (2, 16384), (1, 16383)]
TYPES = [(torch.float32, torch.float32), (torch.bfloat16, torch.bfloat16), (torch.float16, torch.float16), (torch.bfloat16, torch.float32),
         (torch.float16, torch.float32)]


@pytest.mark.parametrize("dtype,wdtype", TYPES)
@pytest.mark.parametrize("rows,cols", SHAPES)
@pytest.mark.parametrize("pad,residual", [(0, False), (0, True), (3, True), (8, False)])
def test_forward_and_backward(rows, cols, pad, residual, dtype, wdtype):
    gen = torch.Generator().manual_seed(rows * 100003 + cols * 17 + pad)
    x = rows_of(rows, cols, pad, dtype, gen, 1.0, 0.3)
    res = rows_of(rows, cols, pad, dtype, gen, 2.0, -0.1) if residual else None
    w = (torch.randn(cols, generator=gen) * 0.2 + 1).to(wdtype).cuda()
    b = (torch.randn(cols, generator=gen) * 0.1).to(wdtype).cuda()
    s, mean, rstd, xh, y, wd, bd = reference(x, res, w, b, 1e-5)
    mag = s.abs().mean(1, keepdim=True) * rstd      # how much the mean's rounding weighs
    got, total, gmean, grstd = S().layer_norm(x, w, b, 1e-5, residual=res)
    check("y", got, y, (xh * wd).abs() + mag * wd.abs() + bd.abs(), 64)
    check("mean", gmean, mean[:, 0], s.abs().mean(1), 32)
    check("rstd", grstd, rstd[:, 0], rstd[:, 0] * (1 + (mag[:, 0] * 27 * EPS) ** 2 / EPS), 32)
    if residual:
        check("sum", total, s, s.abs(), 1)
    else:
        assert total is x
    # the backward pass works on the sum as it was stored
    dy = rows_of(rows, cols, pad, dtype, gen)
    dsum = rows_of(rows, cols, pad, dtype, gen) if residual else None
    sd = total.double()
    xh = (sd - gmean.double()[:, None]) * grstd.double()[:, None]
    e = dy.double() * wd
    c1, c2 = e.mean(1, keepdim=True), (e * xh).mean(1, keepdim=True)
    r = grstd.double()[:, None]
    want = r * (e - c1 - xh * c2) + (0 if dsum is None else dsum.double())
    scale = r * (e.abs() + e.abs().mean(1, keepdim=True) + (xh.abs() + mag) * ((e * xh).abs().mean(1, keepdim=True) + mag * e.abs().mean(1, keepdim=True)))
    dx, dw, db = S().layer_norm_backward(dy, total, gmean, grstd, w, dsum=dsum)
    check("dx", dx, want, scale + (0 if dsum is None else dsum.double().abs()), 128)
    check("dw", dw, (dy.double() * xh).sum(0), (dy.double().abs() * (xh.abs() + mag)).sum(0), 64 + rows // 4)
    check("db", db, dy.double().sum(0), dy.double().abs().sum(0), 64 + rows // 4)
    # the same bits again
    again = S().layer_norm_backward(dy, total, gmean, grstd, w, dsum=dsum)
    for p, q in zip((dx, dw, db), again):
        assert torch.equal(p, q)


def test_many_rows_per_block_and_no_weights():
    gen = torch.Generator().manual_seed(5)
    x = rows_of(20011, 72, 0, torch.float32, gen, 3.0, 1.0)
    s, mean, rstd, xh, y, wd, bd = reference(x, None, None, None, 0.0)
    got, _, m, r = S().layer_norm(x, eps=0.0)
    check("y", got, y, xh.abs() + s.abs().mean(1, keepdim=True) * rstd, 64)
    dy = rows_of(20011, 72, 0, torch.float32, gen)
    dx, dw, db = S().layer_norm_backward(dy, x, m, r)
    check("dw", dw, (dy.double() * xh).sum(0), (dy.double().abs() * (xh.abs() + 1)).sum(0), 64 + 20011 // 4)
    check("db", db, dy.double().sum(0), dy.double().abs().sum(0), 64 + 20011 // 4)


def test_no_rows():
    x = torch.empty(0, 40, device="cuda")
    w = torch.ones(40, device="cuda")
    y, s, m, r = S().layer_norm(x, w, w)
    assert y.shape == (0, 40) and m.shape == (0,)
    dw = torch.full((40,), float("nan"), device="cuda")
    db = torch.full((40,), float("nan"), device="cuda")
    S().layer_norm_backward(x, x, m, r, w, dweight=dw, dbias=db)
    assert float(dw.abs().sum() + db.abs().sum()) == 0.0     # a sum over nothing


def test_constant_rows_large_means_and_bad_rows_stay_apart():
    x = torch.randn(64, 640, generator=torch.Generator().manual_seed(1)).cuda()
    x[3] = 7.25
    x[4] += 4096.0
    x[5, 17] = float("inf")
    x[6, 639] = float("nan")
    y, _, m, r = S().layer_norm(x, eps=1e-5)
    assert float(y[3].abs().max()) == 0.0 and abs(float(r[3]) * 1e-5 ** 0.5 - 1) < 1e-6
    s, mean, rstd, xh, want, _, _ = reference(x[4:5], None, None, None, 1e-5)
    check("row with a large mean", y[4:5], want, xh.abs() + s.abs().mean(1, keepdim=True) * rstd, 64)
    assert torch.isnan(y[5]).any() and torch.isnan(y[6]).any()
    keep = [i for i in range(64) if i not in (5, 6)]
    assert torch.isfinite(y[keep]).all()
    dx, _, _ = S().layer_norm_backward(torch.ones_like(x), x, m, r)
    assert torch.isfinite(dx[keep]).all()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("cols", [96, 1001, 4096])
def test_in_place(cols, dtype):
    gen = torch.Generator().manual_seed(cols)
    x, res = rows_of(37, cols, 0, dtype, gen), rows_of(37, cols, 0, dtype, gen)
    y, s, m, r = S().layer_norm(x, residual=res)
    dy, ds = rows_of(37, cols, 0, dtype, gen), rows_of(37, cols, 0, dtype, gen)
    dx, _, _ = S().layer_norm_backward(dy, s, m, r, dsum=ds)
    x2, res2, dy2 = x.clone(), res.clone(), dy.clone()
    S().layer_norm(x2, residual=res2, out=x2, sum_out=res2)
    assert torch.equal(x2, y) and torch.equal(res2, s)
    S().layer_norm_backward(dy2, s, m, r, dsum=ds, dx=dy2)
    assert torch.equal(dy2, dx)


def test_gradient_against_differences():
    """Directional differences of sum(dy * y), formed in 64 bits from the 32-bit forward pass.  h = 1/64: the third
    derivative leaves below h^2 = 2.4e-4 of the scale, the rounding of y 2 eps / h = 8e-6; bound 1e-3."""
    gen = torch.Generator().manual_seed(9)
    x, dy = rows_of(20, 300, 0, torch.float32, gen), rows_of(20, 300, 0, torch.float32, gen)
    w, b = torch.randn(300, generator=gen).cuda(), torch.randn(300, generator=gen).cuda()
    _, _, m, r = S().layer_norm(x, w, b)
    dx, dw, db = S().layer_norm_backward(dy, x, m, r, w)
    h = 1.0 / 64

    def value(x_, w_, b_):
        return float((S().layer_norm(x_, w_, b_)[0].double() * dy.double()).sum())

    for name, grad, args in (("x", dx, lambda v: (x + v, w, b)), ("w", dw, lambda v: (x, w + v, b)), ("b", db, lambda v: (x, w, b + v))):
        v = torch.randn(grad.shape, generator=gen).cuda() * h
        slope = (value(*args(v)) - value(*args(-v))) / 2
        want = float((grad.double() * v.double()).sum())
        scale = float(grad.double().norm() * v.double().norm())
        assert abs(slope - want) <= 1e-3 * scale, (name, slope, want, scale)


def test_other_stream_and_graph():
    gen = torch.Generator().manual_seed(2)
    x, w = rows_of(200, 512, 0, torch.bfloat16, gen), torch.randn(512, generator=gen).bfloat16().cuda()
    want = S().layer_norm(x, w)[0]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = S().layer_norm(x, w)[0]
    side.synchronize()
    assert torch.equal(got, want)
    out = torch.empty_like(x)
    with torch.cuda.stream(side):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            S().layer_norm(x, w, out=out)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(out, want)
