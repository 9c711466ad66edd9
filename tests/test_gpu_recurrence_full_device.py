"""GPU: the gated recurrence with as many blocks as the device has places for in clusters (33 units of eight blocks on 148
SMs), and one unit more; bounds as in test_gpu_recurrence.py."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from test_gpu_recurrence import check, inputs, reference  # noqa: E402


@pytest.mark.parametrize("N,D", [(1, 1056), (1, 1088), (33, 64), (34, 64), (3, 352)])
@pytest.mark.parametrize("p_done", [0.0, 0.01])
def test_clusters_that_fill_the_device(N, D, p_done):
    from paper_1906_04585_b200 import sequence as S
    T = 2500
    f, x, h0, done, dh, dh_last = inputs(T, N, D, torch.bfloat16, N + D, "time", 0, p_done)
    want = reference(f, x, h0, done, dh, dh_last)
    h, last, states = S.gated_recurrence(f, x, h0, done=done, save=True)
    check("h", h, *want["h"])
    check("h_last", last, *want["h_last"])
    for name, got in zip(("df", "dx", "dh0"), S.gated_recurrence_backward(dh, f, x, states, done=done, dh_last=dh_last)):
        check(name, got, *want[name])
    S.check()
