"""GPU: the filtered draw against the definition, evaluated row by row in 64 bits.

The kernel's weights are 32-bit exponentials of a 32-bit quotient: within 4 units of 2^-23 plus |z| 2^-23 of the 64-bit
ones, below 1e-5 for every weight that matters (|z| < 60).  Where a cut or the draw falls within 1e-5 (relative to the
sum) of a boundary the token may therefore be the one that the definition gives on the boundary's other side; everywhere
else it has to be the definition's.  Log-probabilities: 1e-5 absolute plus one rounding."""
import math

import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

NEAR = 1e-5


def S():
    from paper_1906_04585_b200 import sequence
    return sequence


def rows_answers(l, u, t=1.0, k=0, p=1.0, m=0.0):
    """[(token, logprob), ...] of one row of float64 logits: the definition's answer first, then those it gives when a
    boundary that is near falls on its other side."""
    l = np.where(np.isnan(l), -np.inf, l)
    top = l.max()
    if top == -np.inf:
        return [(-1, -np.inf)]
    if not t > 0:
        return [(int(np.argmax(l)), 0.0)]
    with np.errstate(invalid="ignore", over="ignore"):
        w = np.where(l == top, 1.0, np.where(l == -np.inf, 0.0, np.exp((l - top) / t)))
    ranked = np.argsort(-l, kind="stable")
    if k > 0:
        ranked = ranked[:k]
    exact = set(np.unique(w)) <= {0.0, 1.0}       # sums of whole numbers: both sides decide alike
    wiggle = (0.0,) if exact else (0.0, -NEAR, NEAR)
    answers = []
    for dp in wiggle if p < 1.0 else (0.0,):
        for dm in wiggle if 0 < m < 1.0 else (0.0,):
            order = ranked
            if not p >= 1.0:
                mass = w[order]
                before = np.cumsum(mass) - mass
                order = order[:max(1, int((before < (max(p, 0.0) + dp) * mass.sum()).sum()))]
            if m > 0:
                order = order[w[order] >= min(m * (1 + dm), 1.0)]
            kept = np.sort(order)
            cdf = np.cumsum(w[kept])
            last = int(np.nonzero(w[kept])[0][-1])
            lo, hi = (min(int((cdf <= (u + du) * cdf[-1]).sum()), last) for du in ((0.0, 0.0) if exact else (-NEAR, NEAR)))
            mid = min(int((cdf <= u * cdf[-1]).sum()), last)
            for at in [mid] + list(range(lo, hi + 1)):
                if w[kept[at]] > 0:
                    answers.append((int(kept[at]), math.log(w[kept[at]] / cdf[-1])))
    return answers


def compare(logits, u, t=None, k=None, p=None, m=None):
    R = logits.shape[0]
    dev = [None if a is None else torch.as_tensor(a, dtype=dt).cuda()
           for a, dt in ((u, torch.float32), (t, torch.float32), (k, torch.int32), (p, torch.float32), (m, torch.float32))]
    tok, lp = S().sample(logits, dev[0], dev[1], dev[2], dev[3], dev[4])
    again = S().sample(logits, dev[0], dev[1], dev[2], dev[3], dev[4])
    assert torch.equal(tok, again[0]) and torch.equal(lp, again[1])
    l64 = logits.double().cpu().numpy()
    host = [None if d is None else d.cpu().numpy() for d in dev]
    for r in range(R):
        args = [d[r].item() if d is not None else default for d, default in zip(host[1:], (1.0, 0, 1.0, 0.0))]
        answers = rows_answers(l64[r], float(host[0][r]), *args)
        got, glp = int(tok[r]), float(lp[r])
        fits = [a for a in answers if a[0] == got and (glp == a[1] or abs(glp - a[1]) <= 1e-5 + 2 ** -24 * abs(a[1]))]
        assert fits, (r, got, glp, answers[:4], args)


VOCABS = [1, 2, 18, 32, 33, 255, 257, 1000, 1024, 1025, 5000, 16384, 16385, 32768, 32769, 100003, 131072, 262144]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("vocab", VOCABS)
def test_filters(vocab, dtype):
    R = 24 if vocab > 20000 else 61
    gen = torch.Generator().manual_seed(vocab)
    rng = np.random.default_rng(vocab)
    logits = (torch.randn(R, vocab, generator=gen) * 2.5).to(dtype).cuda()
    u = rng.random(R, dtype=np.float32)
    compare(logits, u)
    t = np.where(rng.random(R) < 0.1, 0.0, rng.uniform(0.3, 2.0, R))
    k = np.where(rng.random(R) < 0.3, 0, np.exp(rng.uniform(0, math.log(2 * vocab), R)).astype(int))
    p = np.where(rng.random(R) < 0.3, 1.0, rng.uniform(0.01, 1.0, R))
    m = np.where(rng.random(R) < 0.5, 0.0, rng.uniform(0.0, 0.3, R))
    compare(logits, u, t=t)
    compare(logits, u, k=k)
    compare(logits, u, p=p)
    compare(logits, u, m=m)
    compare(logits, u, t, k, p, m)


@pytest.mark.parametrize("vocab", [7, 100, 3000, 50000])
def test_ties(vocab):
    """Few distinct values: cuts fall inside runs of equal entries, which stay lowest index first."""
    R = 40
    rng = np.random.default_rng(vocab)
    logits = torch.from_numpy(rng.integers(0, 2, (R, vocab)).astype(np.float32) * 500.0).cuda()     # weights 1 and 0
    logits[:4] = 0.0
    u = rng.random(R, dtype=np.float32)
    for dtype in (torch.float32, torch.bfloat16):
        compare(logits.to(dtype), u, k=rng.integers(1, vocab + 1, R))
        compare(logits.to(dtype), u, p=np.full(R, 0.5))
        compare(logits.to(dtype), u, t=np.zeros(R))
        compare(logits.to(dtype), u, k=np.full(R, max(1, vocab // 3)), p=np.full(R, 0.25), m=np.full(R, 1.0))


@pytest.mark.parametrize("vocab", [1, 5, 31, 700, 4000, 40000])
def test_masked_and_special_rows(vocab):
    gen = torch.Generator().manual_seed(vocab)
    R = 16
    logits = torch.randn(R, vocab, generator=gen).cuda()
    last = vocab - 1
    inf = float("inf")
    logits[0] = -inf                                   # nothing left
    logits[1] = float("nan")
    logits[2] = -inf
    logits[2, last] = 0.5                              # one left, the last
    logits[3] = torch.finfo(torch.float32).min         # masks of the lowest value, everywhere ...
    logits[4] = torch.finfo(torch.float32).min         # ... and all but one
    logits[4, last // 2] = 1.0
    logits[5, last] = inf                              # certain
    logits[6, 0] = inf
    logits[6, last] = inf
    logits[7, last // 2] = float("nan")
    logits[8] = 0.0
    logits[8, ::2] = -0.0
    logits[9] = torch.finfo(torch.float32).max
    logits[10] = -inf
    logits[10, 0] = torch.finfo(torch.float32).min
    u = np.linspace(0.0, 0.9999999, R).astype(np.float32)
    half = np.full(R, 0.5)
    for dtype in (torch.float32, torch.bfloat16):
        x = logits.clone()
        if dtype == torch.bfloat16:      # its own lowest value; float32's would round to -inf
            x[3] = x[4] = torch.finfo(dtype).min
            x[4, last // 2] = 1.0
            x[9] = torch.finfo(dtype).max
            x[10, 0] = torch.finfo(dtype).min
        x = x.to(dtype)
        compare(x, u)
        compare(x, u, t=half)
        compare(x, u, k=np.full(R, 2), p=half, m=np.full(R, 0.01))
        compare(x, u, t=np.zeros(R))


def test_odd_settings():
    """u at and past its ends, filters at and past theirs."""
    logits = torch.randn(12, 300, generator=torch.Generator().manual_seed(3)).cuda()
    last = float(np.nextafter(np.float32(1), np.float32(0)))
    compare(logits, np.array([0.0, last] * 6, np.float32), k=np.array([1, 2, 299, 300, 301, -5, 0, 7, 1, 1, 2, 2]))
    compare(logits, np.full(12, 0.5, np.float32), p=np.array([0.0, -1.0, 1.0, 2.0, 1e-30, 0.999999, 0.5, 0.5, 0.5, 0.5, 0.5, 0.5]))
    compare(logits, np.full(12, 0.5, np.float32), m=np.array([0.0, -1.0, 1.0, 7.0, 1e-30, 0.999999, 0.5, 0.5, 0.5, 0.5, 0.5, 0.5]))
    compare(logits, np.full(12, 0.3, np.float32), t=np.array([0.0, -1.0, 1e-3, 1e3, 1e30, 0.01, 1, 1, 1, 1, 1, 1]))
    # a uniform outside [0, 1) takes the first or the last entry that can be drawn
    tok, _ = S().sample(logits[:3], torch.tensor([1.0, -0.5, float("nan")]).cuda())
    assert tok.tolist() == [299, 0, 0]


def test_row_strides_empty_batches_and_more_rows_than_blocks():
    wide = torch.randn(5000, 40, generator=torch.Generator().manual_seed(8)).cuda()
    u = torch.rand(5000, generator=torch.Generator().manual_seed(9)).cuda()
    a = S().sample(wide[:, 3:36], u)[0]
    b = S().sample(wide[:, 3:36].contiguous(), u)[0]
    assert torch.equal(a, b) and int(a.min()) >= 0 and int(a.max()) < 33
    tok, lp = S().sample(wide[:0], u[:0])
    assert tok.shape == (0,) and lp.shape == (0,)


def test_frequencies():
    """4096 evenly spaced uniforms on one distribution: each token as often as its probability says, within one."""
    logits = torch.randn(1, 18, generator=torch.Generator().manual_seed(2)).cuda().expand(4096, 18)
    u = ((torch.arange(4096) + 0.5) / 4096).cuda()
    tok, lp = S().sample(logits.contiguous(), u)
    want = torch.softmax(logits[0].double(), 0) * 4096
    assert float((torch.bincount(tok.long(), minlength=18) - want).abs().max()) <= 1.0
    assert float((lp.double() - torch.log_softmax(logits[0].double(), 0)[tok.long()]).abs().max()) < 1e-6
