"""GPU: digits of the float32 state that bfloat16 calls in chunks leave, where each entry has one term.

Step j writes value v_j into row j of the state alone, so s_last[j] = g^(steps after j) v_j: a power (its argument, |n log_decay|
units of 2^-24, and an exponential, 2 units in the last place = 4), a product with v held in three pieces (1, and what the third leaves,
1), their sum (2 for a sum that cuts off) and, from chunk to chunk, another power and a product each (|n log_decay| + 4 + 1).  ds0 has a
product with the scale and one with g more (1 and 1 + 4).
"""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

EPS = 2.0 ** -24


@pytest.mark.parametrize("T", [64, 128, 300])
@pytest.mark.parametrize("width", [64, 128])
@pytest.mark.parametrize("first", [0, 40])
def test_one_term_an_entry(first, width, T):
    from paper_1906_04585_b200 import sequence as S
    gen = torch.Generator().manual_seed(T + width)
    rows = min(width, T - first)
    ld = torch.tensor([0.0, -0.0003, -0.0101, -0.2, -1.1])
    H = len(ld)
    v = torch.randn(T, 1, H, width, generator=gen).bfloat16()
    one = torch.zeros(T, 1, H, width)
    for j in range(rows):
        one[first + j, 0, :, j] = 1.0
    one, ld_ = one.bfloat16().cuda(), ld.cuda()
    scale = 0.3
    chunks = (T + 127) // 128
    after = torch.arange(T, dtype=torch.float64)[first:first + rows]
    for name, got, n, factor in (
            ("s_last", S.linear_attention(one, one, v.cuda(), ld_, scale=scale)[1], T - 1 - after, 1.0),
            ("ds0", S.linear_attention_backward(v.cuda(), one, one, one, ld_, scale=scale)[3], after + 1, float(torch.tensor(scale)))):
        power = torch.exp(ld.double().view(H, 1) * n)
        want = factor * power.unsqueeze(-1) * v[first:first + rows, 0].transpose(0, 1).double()
        bound = ((ld.double().abs().view(H, 1) * n) + 4 + 4 + 5 * chunks + 6).unsqueeze(-1) * EPS * want.abs() + 1e-37
        off = (got[0, :, :rows].double().cpu() - want).abs()
        assert (off <= bound).all(), (name, float((off / bound).max()))
        assert float(got[0, :, rows:].abs().max() if rows < width else 0.0) == 0.0
    S.check()
