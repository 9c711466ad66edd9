"""GPU: attention with a memory of fixed size in calls of a few steps, whose state passes through a block once, for narrow
values too, and on both sides of the edge to the longer calls.  Bounds are those of test_gpu_linear_attention.py."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from test_gpu_linear_attention import check_all, inputs  # noqa: E402


def S():
    from paper_1906_04585_b200 import sequence
    return sequence


def shifted(x):
    """The same numbers, contiguous, 4 bytes behind a 16-byte boundary."""
    y = torch.empty(x.numel() + 1, device=x.device)[1:].view(x.shape)
    return y.copy_(x)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("dv", [1, 3, 4, 8, 12, 16, 17, 20, 32])
@pytest.mark.parametrize("dk", [1, 8, 16, 63, 64, 128])
@pytest.mark.parametrize("T,p_done", [(1, 0.0), (5, 0.2), (9, 0.0), (32, 0.05), (33, 0.05)])
def test_narrow_heads(T, p_done, dk, dv, dtype):
    q, k, v, ld, s0, done, do, ds_last = inputs(T, 2, 3, dk, dv, dtype, 100 * T + dk + dv, p_done=p_done)
    for place in (lambda x: x, shifted):
        s0, ds_last = place(s0), place(ds_last)
        got = S().linear_attention(q, k, v, ld, s0, done=done, s_last=place(torch.empty_like(s0)))
        grad = S().linear_attention_backward(do, q, k, v, ld, s0, done=done, ds_last=ds_last)
        S().check()
        check_all(q, k, v, ld, s0, done, dk ** -0.5, do, ds_last, got, grad)


@pytest.mark.parametrize("dk,dv", [(8, 8), (128, 4), (64, 16)])
def test_narrow_heads_in_place(dk, dv):
    q, k, v, ld, s0, done, _, _ = inputs(5, 2, 3, dk, dv, torch.float32, 7, p_done=0.2)
    state, out = s0.clone(), torch.empty(5, 2, 3, dv + 4, device="cuda")[..., :dv]
    got = S().linear_attention(q, k, v, ld, state, done=done, out=out, s_last=state)
    assert got[0] is out and got[1] is state
    check_all(q, k, v, ld, s0, done, dk ** -0.5, got=got)
