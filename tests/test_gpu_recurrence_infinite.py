"""GPU: an infinite state of the gated recurrence stays what it is: a c + b x with a > 0 and c infinite is c, over any
number of steps, however the time axis is cut and however small the product of the gates gets.  What is finite keeps the
bounds of test_gpu_recurrence.py."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from test_gpu_recurrence import check, inputs, reference  # noqa: E402

INF = float("inf")


def S():
    from paper_1906_04585_b200 import sequence
    return sequence


def same(name, got, want):
    got, want = got.double(), want.double()
    assert torch.equal(got, want), "%s: %d of %d differ" % (name, int((got != want).sum()), got.numel())


# one piece, a block, blocks of a cluster, several turns, many sequences (a block each), two pieces a warp
SHAPES = [(1, 2, 40), (12, 2, 40), (16, 1, 64), (17, 2, 40), (90, 2, 40), (300, 2, 40), (1500, 2, 40), (5000, 1, 64), (150, 300, 40), (700, 40, 130)]


@pytest.mark.parametrize("gates", ["mixed", "half", "shut"])
@pytest.mark.parametrize("flags", [None, "none set", "some"])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("T,N,D", SHAPES)
def test_infinities_stay(T, N, D, dtype, flags, gates):
    f, x, h0, _, dh, dh_last = inputs(T, N, D, dtype, T + N + D, "time", 0, 0.0)
    if gates == "half":        # 150 of them leave float32's range
        f = torch.zeros_like(f)
    elif gates == "shut":      # two of them do
        f = torch.full_like(f, -60.0)
    done = None if flags is None else torch.zeros(T, N, dtype=torch.bool, device="cuda")
    cut = T // 3
    if flags == "some":
        done[cut, 0] = True
    t = T // 2
    clean = reference(f, x, h0, done, dh, dh_last)
    # channel 3: infinite from the start, 5: minus that, 9 of the last sequence: from step t on
    h0, x = h0.clone(), x.clone()
    h0[0, 3], h0[0, 5], x[t, N - 1, 9] = INF, -INF, INF
    h, last, states = S().gated_recurrence(f, x, h0, done=done, save=True)
    want_h, want_last = clean["h"][0].clone(), clean["h_last"][0].clone()
    end = cut + 1 if flags == "some" else T
    want_h[:end, 0, 3], want_h[:end, 0, 5] = INF, -INF
    want_h[t:end if N == 1 and t < end else T, N - 1, 9] = INF
    if flags != "some":
        want_last[0, 3], want_last[0, 5] = INF, -INF
    if flags != "some" or N > 1 or t > cut:
        want_last[N - 1, 9] = INF
    if flags == "some" and cut == T - 1:
        want_last[0] = 0.0
    far = torch.isinf(want_h)
    same("h where it is infinite", h[far], want_h[far])
    check("h", h[~far], want_h[~far], clean["h"][1][~far])
    far = torch.isinf(want_last)
    same("h_last where it is infinite", last[far], want_last[far])
    check("h_last", last[~far], want_last[~far], clean["h_last"][1][~far])

    # backwards, from a finite forward pass: q from the last step or from step t
    f, x, h0 = f, inputs(T, N, D, dtype, T + N + D, "time", 0, 0.0)[1], inputs(T, N, D, dtype, T + N + D, "time", 0, 0.0)[2]
    _, _, states = S().gated_recurrence(f, x, h0, done=done, save=True)
    dh, dh_last = dh.clone(), dh_last.clone()
    dh_last[0, 3], dh_last[0, 5], dh[t, N - 1, 9] = INF, -INF, INF
    df, dx, dh0 = S().gated_recurrence_backward(dh, f, x, states, done=done, dh_last=dh_last)
    want, want0 = clean["dx"][0].clone(), clean["dh0"][0].clone()
    begin = cut + 1 if flags == "some" else 0
    want[begin:, 0, 3], want[begin:, 0, 5] = INF, -INF
    want[(begin if N == 1 and begin <= t else 0):t + 1, N - 1, 9] = INF
    if flags != "some":
        want0[0, 3], want0[0, 5] = INF, -INF
    if flags != "some" or N > 1 or t <= cut:
        want0[N - 1, 9] = INF
    far = torch.isinf(want)
    same("dx where it is infinite", dx[far], want[far])
    check("dx", dx[~far], want[~far], clean["dx"][1][~far])
    assert not torch.isnan(df[far]).all() and not torch.isfinite(df[far]).any()
    check("df", df[~far], clean["df"][0][~far], clean["df"][1][~far])
    far = torch.isinf(want0)
    same("dh0 where it is infinite", dh0[far], want0[far])
    check("dh0", dh0[~far], want0[~far], clean["dh0"][1][~far])
