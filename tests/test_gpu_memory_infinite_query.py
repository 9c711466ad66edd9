"""GPU: an infinite query (or gradient of o) of the attention memory makes its own step infinite, with the signs of the state that
it reads, and no other.  The rest keeps the bounds of test_gpu_linear_attention.py."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from test_gpu_linear_attention import Pass, check, inputs  # noqa: E402


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("T", [5, 33, 130, 700])
@pytest.mark.parametrize("width", [64, 128])
def test_an_infinite_query(width, T, dtype):
    from paper_1906_04585_b200 import sequence as S
    q, k, v, _, s0, _, do, _ = inputs(T, 2, 3, width, width, dtype, T + width)
    # values of both signs beside a state that stays positive
    q, k, s0, ld = q.abs() + 0.125, k.abs() + 0.125, s0 + 1000.0, torch.full((3,), -1e-3, device="cuda")
    t = T // 2
    bad = q.clone()
    bad[t, 1, 2, 3] = float("inf")
    o, last = S.linear_attention(bad, k, v, ld, s0, scale=0.25)
    assert (o[t, 1, 2] == float("inf")).all()
    keep = torch.ones_like(o, dtype=torch.bool)
    keep[t, 1, 2] = False
    p = Pass(q, k, v, ld, None, s0, True)
    check("o elsewhere", o[keep], 0.25 * p.o[keep], 0.25 * p.a[keep], 0.25 * p.e[keep], width, dtype)
    check("s_last", last, p.X, p.A, p.E, 0, dtype, state=True)
    worse = do.clone()
    worse[t, 1, 2, 3] = -float("inf")
    dq = S.linear_attention_backward(worse, q, k, v, ld, s0, scale=0.25)[0]
    assert (dq[t, 1, 2] == -float("inf")).all()
    p = Pass(do, v, k, ld, None, s0.transpose(-1, -2), True)
    check("dq elsewhere", dq[keep], 0.25 * p.o[keep], 0.25 * p.a[keep], 0.25 * p.e[keep], width, dtype)
    S.check()
