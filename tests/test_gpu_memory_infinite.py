"""GPU: an infinite entry of the attention memory stays what it is: g X + k v with g > 0 and X infinite is X, over any number of
steps, however the time axis is cut and however small the power of g gets.  A head that keeps nothing (g = 0) keeps no infinity
either.  What is finite keeps the bounds of test_gpu_linear_attention.py, whose 64-bit evaluation has the infinities too."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

import test_gpu_linear_attention as memory  # noqa: E402
from test_gpu_linear_attention import check_all, inputs  # noqa: E402

INF = float("inf")


@pytest.fixture(autouse=True)
def infinities_are_compared(monkeypatch):
    """What is infinite in 64 bits has to be that; the rest goes to the bounds."""
    bounds = memory.check

    def check(name, got, want, absolute, running, width, dtype, state=False):
        want, absolute, running = (torch.where(torch.isnan(absolute), 0.0, x) for x in (want, absolute, running))      # dropped: 0 times an infinity there
        far = torch.isinf(want)
        assert not torch.isnan(want).any()
        assert torch.equal(got[far].double(), want[far]), "%s: %d of %d infinities are others" % (name, int((got[far].double() != want[far]).sum()), int(far.sum()))
        bounds(name, got[~far], want[~far], absolute[~far], running[~far], width, dtype, state)

    monkeypatch.setattr(memory, "check", check)
DECAYS = [0.0, -0.01, -0.6, -4.0]      # the last leaves float32's range within 32 steps


def S():
    from paper_1906_04585_b200 import sequence
    return sequence


def made(T, N, dtype, seed, flags, dk=64, dv=64):
    """Queries and keys positive and no value 0, so that an infinite entry makes all it enters infinite of one sign."""
    q, k, v, _, s0, _, do, ds_last = inputs(T, N, len(DECAYS), dk, dv, dtype, seed)
    q, k = q.abs() + 0.125, k.abs() + 0.125
    v, do = (torch.where(x.abs() < 0.0625, torch.full_like(x, 0.0625), x) for x in (v, do))
    done = None if flags is None else torch.zeros(T, N, dtype=torch.bool, device="cuda")
    if flags == "some":
        done[T // 3, 0] = True
    return q, k, v, torch.tensor(DECAYS, device="cuda"), s0, done, do, ds_last


# one passage of the state, step by step or by a chunk, several, pieces of the time axis
LENGTHS = [1, 2, 5, 32, 33, 90, 129, 300, 1500, 5000]


@pytest.mark.parametrize("flags", [None, "none set", "some"])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("T", LENGTHS)
def test_infinities_stay(T, dtype, flags):
    N = 2
    q, k, v, ld, s0, done, do, ds_last = made(T, N, dtype, T, flags)
    scale = 0.25
    # from the given state, and from a value in the middle
    first, bad = s0.clone(), v.clone()
    first[0, :, 3, 2], first[0, :, 5, 7], bad[T // 2, N - 1, :, 9] = INF, -INF, INF
    got = S().linear_attention(q, k, bad, ld, first, done=done, scale=scale)
    S().check()
    if flags is None:
        assert torch.isinf(got[1][0, :, 3, 2]).all() and torch.isinf(got[1][N - 1, :, :, 9]).all()
    check_all(q, k, bad, ld, first, done, scale, got=got)
    # the same, the state in place
    state = first.clone()
    o, _ = S().linear_attention(q, k, bad, ld, state, done=done, scale=scale, s_last=state)
    assert torch.equal(o, got[0]) and torch.equal(state, got[1])
    # backwards: from the given gradient of the last state, and from a gradient in the middle
    last, worse = ds_last.clone(), do.clone()
    last[0, :, 3, 2], last[0, :, 5, 7], worse[T // 2, N - 1, :, 9] = INF, -INF, INF
    grad = S().linear_attention_backward(worse, q, k, v, ld, s0, done=done, scale=scale, ds_last=last)
    S().check()
    check_all(q, k, v, ld, s0, done, scale, worse, last, got_grad=grad)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("T", [1, 5, 33, 300, 1500])
def test_a_head_that_keeps_nothing_keeps_no_infinity(T, dtype):
    q, k, v, _, s0, _, do, ds_last = made(T, 2, dtype, T, None)
    ld = torch.full((len(DECAYS),), -INF, device="cuda")
    s0, ds_last = torch.full_like(s0, INF), torch.full_like(ds_last, -INF)
    o, last = S().linear_attention(q, k, v, ld, s0)
    check_all(q, k, v, ld, torch.zeros_like(s0), None, 64 ** -0.5, got=(o, last))
    grad = S().linear_attention_backward(do, q, k, v, ld, None, ds_last=ds_last)
    assert float(grad[3].abs().max()) == 0.0
    assert not torch.isfinite(grad[1][-1]).any() and not torch.isfinite(grad[2][-1]).any()      # the last step sees it
    assert torch.isfinite(grad[0]).all() and torch.isfinite(grad[1][:-1]).all() and torch.isfinite(grad[2][:-1]).all()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("T", [1, 5, 33, 300, 1500])
@pytest.mark.parametrize("dk,dv", [(40, 24), (33, 17), (1, 100), (100, 1), (5, 8)])
def test_infinities_beside_the_edge_of_a_head(dk, dv, T, dtype):
    """Heads that leave places of a block empty: 0 there times an infinite entry of k, v or do is not added to what is there."""
    q, k, v, ld, s0, _, do, ds_last = made(T, 2, dtype, T + dk, None, dk, dv)
    v, do = v.abs(), do.abs()      # one sign for all that an infinite key or query enters
    s0, ds_last = s0.abs(), ds_last.abs()
    t, (c, d) = T // 2, (dk // 2, dv // 2)
    bad_v, bad_k = v.clone(), k.clone()
    bad_v[t, 0, :, d], bad_k[t, 1, :, c] = INF, INF
    check_all(q, bad_k, bad_v, ld, s0, None, 0.25, got=S().linear_attention(q, bad_k, bad_v, ld, s0, scale=0.25))
    bad_do, bad_q = do.clone(), q.clone()
    bad_do[t, 0, :, d], bad_q[t, 1, :, c] = INF, INF
    grad = S().linear_attention_backward(bad_do, bad_q, k, v, ld, s0, scale=0.25, ds_last=ds_last)
    S().check()
    check_all(bad_q, k, v, ld, s0, None, 0.25, bad_do, ds_last, got_grad=grad)
