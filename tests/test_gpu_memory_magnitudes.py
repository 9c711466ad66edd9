"""GPU: attention with a memory of fixed size in float16 whose episodes, steps or channels differ in magnitude by far: what a step
gives depends on what it sees, not on the largest values beside it.  Bounds are those of test_gpu_linear_attention.py."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from test_gpu_linear_attention import check_all, inputs  # noqa: E402


@pytest.mark.parametrize("width", [64, 128])
@pytest.mark.parametrize("what", ["queries", "keys", "queries and keys", "values", "keys and values"])
@pytest.mark.parametrize("power", [4, 8, 12])
@pytest.mark.parametrize("T", [250, 700])
def test_episodes_of_many_magnitudes(T, power, what, width):
    from paper_1906_04585_b200 import sequence as S
    q, k, v, ld, s0, _, do, ds_last = inputs(T, 2, 3, width, width, torch.float16, T + power, p_done=0.0)
    done = torch.zeros(T, 2, dtype=torch.uint8, device="cuda")
    done[29::40] = 1
    # every other episode of 40 steps larger by 2^power, per operand
    size = torch.exp2(power * (((torch.arange(T, device="cuda") + 10) // 40) % 2).float()).half().view(T, 1, 1, 1)
    q, k, v = (x * size if any(name in what for name in names) else x for x, names in ((q, ["queries"]), (k, ["keys"]), (v, ["values"])))
    scale = 2.0 ** -(6 + power)
    got = S.linear_attention(q, k, v, ld, s0, done=done, scale=scale)
    grad = S.linear_attention_backward(do, q, k, v, ld, s0, done=done, scale=scale, ds_last=ds_last)
    S.check()
    check_all(q, k, v, ld, s0, done, scale, do, ds_last, got, grad)


@pytest.mark.parametrize("power", [6, 10])
@pytest.mark.parametrize("T", [250, 700])
def test_steps_that_grow(T, power):
    """Magnitudes rise within every chunk: what early steps see is small."""
    from paper_1906_04585_b200 import sequence as S
    q, k, v, ld, s0, _, do, ds_last = inputs(T, 2, 3, 64, 64, torch.float16, T + power)
    size = torch.exp2(power * torch.linspace(0, 1, T, device="cuda")).half().view(T, 1, 1, 1)
    q, k, s0 = q * size, k * size, s0 * 0
    scale = 2.0 ** -(6 + power)
    got = S.linear_attention(q, k, v, ld, s0, scale=scale)
    S.check()
    check_all(q, k, v, ld, s0, None, scale, got=got)
