"""GPU: logits before a draw against the definition in 64 bits.

Five float32 operations (quotient or product, two products and differences of the penalties, the bias), each off by eps = 2^-24
of what it gives, which is at most the sum of the absolute values M of all that enters; a list of n biases for one entry adds n
more; then one rounding to the element type.  Bound: (n + 8) eps M + u |result|.  What is crossed out is -inf exactly."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

EPS = 2.0 ** -24
U = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}


def S():
    from paper_1906_04585_b200 import sequence
    return sequence


def reference(x, history=None, lengths=None, repetition=None, frequency=None, presence=None, bias_ids=None, bias_values=None, mask=None):
    """(result, bound before the last rounding), row by row."""
    R, V = x.shape
    y, m = x.double(), torch.zeros(R, V, dtype=torch.float64, device=x.device)
    m += torch.where(torch.isfinite(y), y.abs(), 0.0)
    n = torch.zeros_like(m)
    for r in range(R):
        if history is not None:
            h = history[r] if lengths is None else history[r, :max(0, int(lengths[r]))]
            h = h[(h >= 0) & (h < V)].long()
            c = torch.bincount(h, minlength=V).double()
            rep, fre, pre = (d if t is None else float(t[r]) for t, d in ((repetition, 1.0), (frequency, 0.0), (presence, 0.0)))
            hit = c > 0
            y[r] = torch.where(hit, torch.where(y[r] > 0, y[r] / rep, y[r] * rep) - fre * c - pre, y[r])
            m[r] += torch.where(hit, torch.where(torch.isfinite(x[r].double()), x[r].double().abs(), 0.0) * max(rep, 1 / rep) + abs(fre) * c + abs(pre), 0.0)
        if bias_ids is not None:
            ok = (bias_ids[r] >= 0) & (bias_ids[r] < V)
            y[r].index_add_(0, bias_ids[r][ok].long(), bias_values[r][ok].double())
            m[r].index_add_(0, bias_ids[r][ok].long(), bias_values[r][ok].double().abs().nan_to_num(0, 0, 0))
            n[r].index_add_(0, bias_ids[r][ok].long(), torch.ones(int(ok.sum()), dtype=torch.float64, device=x.device))
    if mask is not None:
        at = torch.arange(V, device=x.device)
        y = torch.where((mask[:, at // 32] >> (at % 32)) & 1 != 0, y, -float("inf"))
    return y, (n + 8) * EPS * m


def check(got, want, err):
    # a value past the type's largest number is infinite there (float32's own lowest value, multiplied, among them)
    want = torch.where(torch.isinf(got) & (want.abs() + err > torch.finfo(got.dtype).max), want.sign() * float("inf"), want)
    fine = torch.isfinite(want)
    assert torch.equal(torch.isnan(got), torch.isnan(want))
    rest = ~fine & ~torch.isnan(want)
    assert torch.equal(got[rest].double(), want[rest])
    off = (got.double() - want)[fine].abs()
    bound = (U[got.dtype] * want.abs() + err * 1.01 + 2.0 ** -25)[fine] if got.dtype == torch.float16 else (U[got.dtype] * want.abs() + err * 1.01 + 1e-37)[fine]
    assert (off <= bound).all(), float((off / bound).max())


def inputs(R, V, W, B, dtype, seed, masked=True, pad=0):
    gen = torch.Generator().manual_seed(seed)
    a = {"logits": (torch.randn(R, V + pad, generator=gen) * 3).to(dtype).cuda()[:, :V]}
    if W:
        a["history"] = (V * torch.rand(R, W, generator=gen) ** 3).to(torch.int32).clamp(max=V - 1).cuda()
        a["history"][torch.rand(R, W, generator=gen).cuda() < 0.1] = -1
        a["lengths"] = torch.randint(0, W + 1, (R,), generator=gen).to(torch.int32).cuda()
        a["repetition"] = (0.8 + torch.rand(R, generator=gen)).cuda()
        a["frequency"], a["presence"] = ((torch.rand(R, generator=gen) - 0.2).cuda() for _ in range(2))
    if B:
        a["bias_ids"] = torch.randint(-1, V, (R, B), generator=gen).to(torch.int32).cuda()
        a["bias_values"] = (torch.randn(R, B, generator=gen) * 4).cuda()
    if masked:
        a["mask"] = torch.randint(-2 ** 31, 2 ** 31, (R, (V + 31) // 32), generator=gen).to(torch.int32).cuda()
    return a


def run(a, **kw):
    a = dict(a)
    return S().adjust_logits(a.pop("logits"), **a, **kw)


def want(a):
    a = dict(a)
    return reference(a.pop("logits"), **a)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("R,V,W,B,masked,pad", [
    (1, 1, 1, 1, True, 0), (5, 18, 0, 0, True, 0), (5, 18, 7, 3, True, 6), (3, 33, 100, 0, False, 0), (2, 1000, 0, 40, False, 24), (4, 4096, 300, 20, True, 0),
    (2, 16384, 50, 5, True, 0), (2, 16385, 50, 5, True, 0), (3, 40007, 2000, 300, True, 1), (1, 131072, 5000, 0, True, 0), (2, 50000, 0, 0, True, 0),
    (300, 64, 20, 2, True, 0), (2, 131, 3, 4095, False, 0), (2, 20000, 12000, 7, True, 0), (3, 9001, 0, 4095, True, 7), (2, 30000, 10000, 900, False, 0)])
def test_against_the_definition(R, V, W, B, masked, pad, dtype):
    a = inputs(R, V, W, B, dtype, R + V + W, masked, pad)
    check(run(a), *want(a))


def test_parts_may_be_left_out():
    a = inputs(4, 300, 60, 8, torch.float32, 3)
    for names in (("history",), ("history", "lengths"), ("history", "repetition"), ("history", "lengths", "frequency"), ("history", "presence", "mask"),
                  ("bias_ids", "bias_values"), ("mask",), ()):
        b = {k: v for k, v in a.items() if k in names + ("logits",)}
        check(run(b), *want(b))


def test_the_same_id_again_and_again():
    """Every token and every bias is the same entry; sums of a bias come in the order of the list, the same bits every time."""
    a = inputs(3, 500, 1000, 200, torch.float32, 4)
    a["history"][:] = 77
    a["bias_ids"][:] = 77
    first = run(a)
    check(first, *want(a))
    for _ in range(5):
        assert torch.equal(first, run(a))
    total = torch.zeros(3, device="cuda")
    for j in range(200):
        total = total + a["bias_values"][:, j] if j else a["bias_values"][:, 0]
    b = {k: v for k, v in a.items() if k in ("logits", "bias_ids", "bias_values")}
    assert torch.equal(run(b)[:, 77], a["logits"][:, 77] + total)


def test_ids_and_lengths_out_of_range_count_nowhere():
    a = inputs(4, 20000, 12, 6, torch.float32, 5)
    odd = torch.tensor([-1, -2 ** 31, 2 ** 31 - 1, 20000, 16384 - 2 ** 31, 32768], dtype=torch.int32, device="cuda")
    a["history"][:, ::2], a["bias_ids"][0] = odd, odd
    a["lengths"] = torch.tensor([-5, 2 ** 31 - 1, 12, 0], dtype=torch.int32, device="cuda")
    b = dict(a, lengths=torch.tensor([0, 12, 12, 0], dtype=torch.int32, device="cuda"))
    check(run(a), *want(b))


def test_one_mask_for_all_rows_and_masks_that_leave_nothing():
    a = inputs(6, 100, 0, 0, torch.bfloat16, 6)
    shared = a["mask"][:1]
    check(S().adjust_logits(a["logits"], mask=shared), *reference(a["logits"], mask=shared.expand(6, -1)))
    a["mask"][2] = 0
    y = run(a)
    assert bool((y[2] == -float("inf")).all())
    assert int(S().sample(y, torch.zeros(6, device="cuda"))[0][2]) == -1


def test_infinities_and_nan():
    a = inputs(4, 64, 10, 4, torch.float32, 7)
    a["logits"] = a["logits"].clone()
    a["logits"][0, :20], a["logits"][1, :20], a["logits"][2, :20] = float("inf"), -float("inf"), float("nan")
    a["logits"][3] = torch.finfo(torch.float32).min
    a["bias_values"][0, 0], a["bias_values"][1, 1] = float("inf"), -float("inf")
    check(run(a), *want(a))


@pytest.mark.parametrize("V,masked", [(1000, True), (20000, True), (20000, False), (8193, True)])
def test_in_place_and_strided(V, masked):
    a = inputs(7, V, 30, 4, torch.bfloat16, 8, masked, pad=40)
    y, err = want(a)
    got = run(a, out=a["logits"])
    assert got is a["logits"]
    check(got, y, err)


def test_captured_with_the_draw():
    """Adjust and draw in one graph, replayed over other logits and a grown history."""
    a = inputs(16, 5000, 40, 6, torch.float32, 9)
    a["lengths"][:] = 3
    u = torch.rand(16, device="cuda")
    run(a)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y = run(a)
        token, logp = S().sample(y, u)
    a["logits"].mul_(0.5)
    a["lengths"][:] = 40
    graph.replay()
    torch.cuda.synchronize()
    check(y, *want(a))
    t2, l2 = S().sample(run(a), u)
    assert torch.equal(token, t2) and torch.equal(logp, l2)
    allowed = (a["mask"].gather(1, (t2 // 32).long().unsqueeze(1)) >> (t2 % 32).unsqueeze(1)) & 1
    assert bool((allowed != 0).all())
