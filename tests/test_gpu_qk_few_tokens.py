"""GPU: gradients of the norm and rotation where a few tokens have many heads, which are shared out over the device and whose sums of
the weights' gradients come from as many blocks.  Bounds are those of test_gpu_qk_norm_rotary.py."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from test_gpu_qk_norm_rotary import check, inputs  # noqa: E402


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("n,hq,hk,dim,pairs", [(1, 300, 7, 64, 32), (1, 5000, 1, 128, 64), (16, 32, 8, 128, 64), (3, 70, 70, 75, 20), (700, 9, 3, 256, 100), (2, 1, 1, 8, 4)])
def test_few_tokens_of_many_heads(n, hq, hk, dim, pairs, dtype):
    from paper_1906_04585_b200 import sequence as S
    q, k, wq, wk, positions, inv_freq, dq, dk = inputs(n, hq, hk, dim, pairs, dtype, torch.float32, n + hq, "flat")
    first = None
    for _ in range(3):
        g = S.qk_norm_rotary_backward(dq, dk, q, k, positions, inv_freq, wq, wk)
        check(q, wq, positions, inv_freq, 1e-6, False, None, dq, g[0], g[2])
        check(k, wk, positions, inv_freq, 1e-6, False, None, dk, g[1], g[3])
        first = first or g
        assert all(torch.equal(a, b) for a, b in zip(first, g))
