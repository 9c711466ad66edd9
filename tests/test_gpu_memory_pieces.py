"""GPU: attention with a memory of fixed size over long sequences in float16, whose pieces of the time axis are several chunks
long and whose chunks differ in magnitude, so that each has a power of two of its own.  Bounds are those of
test_gpu_linear_attention.py."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from test_gpu_linear_attention import check_all, inputs  # noqa: E402


def S():
    from paper_1906_04585_b200 import sequence
    return sequence


@pytest.mark.parametrize("T,N,H,d", [(8192, 2, 8, 64), (3000, 8, 20, 64), (4096, 2, 8, 128)])
def test_chunks_of_many_magnitudes(T, N, H, d):
    """16 units of 64 chunks: pieces of 8, whose own states come first; and 160 units, which are not cut."""
    q, k, v, ld, s0, done, do, ds_last = inputs(T, N, H, d, d, torch.float16, T, p_done=0.001)
    size = torch.exp2(((torch.arange(T, device="cuda") // 128) * 7 % 5 - 2).float()).half().view(T, 1, 1, 1)
    v, k = v * size, k * size.flip(0)
    got = S().linear_attention(q, k, v, ld, s0, done=done)
    grad = S().linear_attention_backward(do, q, k, v, ld, s0, done=done, ds_last=ds_last)
    S().check()
    check_all(q, k, v, ld, s0, done, d ** -0.5, do, ds_last, got, grad)
    for _ in range(20):
        again = S().linear_attention(q, k, v, ld, s0, done=done)
        assert torch.equal(again[0], got[0]) and torch.equal(again[1], got[1])
