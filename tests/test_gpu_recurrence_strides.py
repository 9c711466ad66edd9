"""GPU: the stride of an axis of one step, or of one sequence, says nothing: any value gives the same bits."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


def S():
    from paper_1906_04585_b200 import sequence
    return sequence


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("shape,strides", [((1, 5, 64), (1 << 30, 64, 1)), ((1, 5, 64), ((1 << 33) + 1, 64, 1)), ((1, 5, 64), (0, 64, 1)),
                                           ((40, 1, 64), (64, (1 << 40) + 1, 1)), ((1, 1, 64), (3, 5, 1))])
def test_strides_of_axes_of_one(shape, strides, dtype):
    T, N, D = shape
    gen = torch.Generator(device="cuda").manual_seed(T)
    f, x, dh = (torch.randn(shape, device="cuda", generator=gen).to(dtype) for _ in range(3))
    h0, done = torch.randn(N, D, device="cuda", generator=gen), torch.zeros(T, N, dtype=torch.bool, device="cuda")
    done[0, 0] = True

    def strange(t, s=strides):
        return t.as_strided(t.shape, s[:t.dim()])

    h, last, states = S().gated_recurrence(f, x, h0, done=done, save=True)
    grads = S().gated_recurrence_backward(dh, f, x, states, done=done, dh_last=h0)
    flags = strange(done, tuple(a if n == 1 else b for n, a, b in zip(done.shape, strides, done.stride())))
    for save in (False, True):
        got = S().gated_recurrence(strange(f), strange(x), h0, done=flags, out=strange(torch.empty_like(x)), save=save)
        assert torch.equal(got[0], h) and torch.equal(got[1], last)
    got = S().gated_recurrence_backward(strange(dh), strange(f), strange(x), states, done=flags, dh_last=h0, df=strange(torch.empty_like(f)),
                                        dx=strange(torch.empty_like(x)))
    assert all(torch.equal(a, b) for a, b in zip(got, grads))
