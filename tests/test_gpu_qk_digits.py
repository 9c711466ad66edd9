"""GPU: digits of the float32 norm and rotation where each part shows by itself.

Sine and cosine: pairs (2, 0) beside as many entries that the norm makes exact (mean of squares 1), so a pair becomes (2 cos f, 2 sin
f) with no rounding but theirs.  The angle is a fraction of a turn in 64 bits, the functions are off by a unit in the last place (2^-23
at most) each, what the fraction loses on its way to 32 bits is put right to first order (a product and a sum, 2^-24 each, and
(pi 2^-25)^2 / 2 left, 4e-15): within 2^-22 of the value itself, near their zeros too, and 1e-14.

The norm: one entry x among dim becomes sqrt(dim).  The square is rounded (2^-24, half of which stays), its quotient by dim is exact for
powers of two, a correctly rounded root's reciprocal adds 2^-24, and the product with x 2^-24: within 2.5 of them.
"""
import math

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.mark.parametrize("dim,interleaved", [(64, False), (64, True), (128, False), (36, True)])
def test_sine_and_cosine(dim, interleaved):
    from paper_1906_04585_b200 import sequence as S
    n = 4096
    pairs = dim // 4      # a quarter of the entries is 2: the mean of their squares is 1
    gen = torch.Generator().manual_seed(dim)
    x = torch.zeros(n, 1, dim)
    if interleaved:
        x[..., 0:2 * pairs:2] = 2.0
    else:
        x[..., :pairs] = 2.0
    positions = torch.randint(-1 << 20, 1 << 20, (n,), generator=gen).to(torch.int32)
    inv_freq = torch.pow(10000.0, -torch.arange(pairs, dtype=torch.float64) / pairs).float()
    # angles next to multiples of a quarter turn, where sine or cosine is small
    near = torch.arange(pairs) % 2 == 0
    inv_freq[near] = (math.pi / 2 * (1 + torch.arange(pairs)[near])).float()
    y = S.qk_norm_rotary(x.cuda(), x.cuda(), positions.cuda(), inv_freq.cuda(), eps=0.0, interleaved=interleaved)[0].cpu().double()
    f = positions.double().unsqueeze(1) * inv_freq.double()
    c, s = (y[:, 0, 0:2 * pairs:2], y[:, 0, 1:2 * pairs:2]) if interleaved else (y[:, 0, :pairs], y[:, 0, pairs:2 * pairs])
    # the angle itself in 64 bits: a product and a multiple of 2 pi, 2^-52 of it
    angle = f.abs() * 2.0 ** -51
    for got, want in ((c, torch.cos(f)), (s, torch.sin(f))):
        bound = 2 * (2.0 ** -22 * want.abs() + angle + 1e-14)
        assert ((got - 2 * want).abs() <= bound).all(), float(((got - 2 * want).abs() / bound).max())


@pytest.mark.parametrize("dim", [8, 64, 128, 256])
def test_norm_of_one_entry(dim):
    from paper_1906_04585_b200 import sequence as S
    gen = torch.Generator().manual_seed(dim)
    n = 20000
    x = torch.zeros(n, 1, dim)
    x[..., dim // 2] = torch.exp2(6 * torch.rand(n, 1, generator=gen) - 3)
    positions, inv_freq = torch.zeros(n, dtype=torch.int32, device="cuda"), torch.empty(0, device="cuda")
    y = S.qk_norm_rotary(x.cuda(), x.cuda(), positions, inv_freq, eps=0.0)[0].cpu().double()[..., dim // 2]
    off = (y / math.sqrt(dim) - 1).abs() * 2.0 ** 24
    assert off.max() <= 2.5 * 1.0001, float(off.max())
