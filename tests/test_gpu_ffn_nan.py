"""GPU: a NaN in one weight of the gated feed-forward block shows in everything that is computed from it, whatever the
activation, and in nothing else.  Elements without a NaN among their terms are compared as bits with a call on clean
weights."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


def S():
    from paper_1906_04585_b200 import sequence
    return sequence


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("kind", ["silu", "gelu", "relu"])
@pytest.mark.parametrize("M", [3, 100, 300])      # few rows, few rows at their widest, pairs of SMs
def test_a_nan_weight_shows(M, kind, dtype):
    D, F, unit = 136, 200, 77
    gen = torch.Generator().manual_seed(M)
    x, wg, wu, wd, dy = ((torch.randn(n, m, generator=gen) * s).to(dtype).cuda()
                         for n, m, s in ((M, D, 1.0), (F, D, D ** -0.5), (F, D, D ** -0.5), (D, F, F ** -0.5), (M, D, 1.0)))
    clean_y, saved = S().gated_ffn(x, wg, wu, wd, kind, save=True)
    clean = S().gated_ffn_backward(dy, x, wg, wu, wd, saved, kind)
    assert all(torch.isfinite(t).all() for t in (clean_y,) + clean)
    bad = wg.clone()
    bad[unit, 5] = float("nan")
    y, _ = S().gated_ffn(x, bad, wu, wd, kind)
    assert torch.isnan(y).all()                                         # every row has unit 77's product among its terms
    y, saved = S().gated_ffn(x, bad, wu, wd, kind, save=True)
    assert torch.isnan(y).all()
    dx, dw_gate, dw_up, dw_down = S().gated_ffn_backward(dy, x, bad, wu, wd, saved, kind)
    others = [i for i in range(F) if i != unit]
    assert torch.isnan(dx).all()
    for got, want in ((dw_gate, clean[1]), (dw_up, clean[2])):          # dg and du of the unit, in every row
        assert torch.isnan(got[unit]).all() and torch.equal(got[others], want[others])
    assert torch.isnan(dw_down[:, unit]).all() and torch.equal(dw_down[:, others], clean[3][:, others])
