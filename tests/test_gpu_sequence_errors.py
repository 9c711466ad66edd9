"""GPU: what the torch front end of the sequence-policy operators says when a call cannot be done, the same from its
compiled and its Python part."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


def S():
    from paper_1906_04585_b200 import sequence
    return sequence


@pytest.mark.parametrize("save", [False, True])      # False: compiled, True: Python
def test_results_that_do_not_fit_are_out_of_memory(save):
    """Inputs that share one row of memory, results of 4 TB: the allocation fails, nothing is launched."""
    row = torch.zeros(512, device="cuda").expand(1 << 21, 1024, 512)
    with pytest.raises(torch.cuda.OutOfMemoryError):
        S().gated_recurrence(row, row, save=save)
    few = torch.zeros(3, 2, 8, device="cuda")
    assert float(S().gated_recurrence(few, few, save=save)[0].abs().max()) == 0.0


def test_sizes_past_32_bits_are_refused():
    """2^32 + 32 columns are not 32."""
    x = torch.empty(1, (1 << 32) + 32, dtype=torch.bfloat16, device="cuda")
    stat, u = torch.ones(1, device="cuda"), torch.zeros(1, device="cuda")
    for call in (lambda: S().layer_norm(x), lambda: S().layer_norm_backward(x, x, stat, stat, dx=x, dweight=u, dbias=u), lambda: S().sample(x, u),
                 lambda: S().gated_ffn(x, x, x, x.T)):
        with pytest.raises(ValueError, match="too large"):
            call()
