"""GPU: the operators together - a policy that acts step by step and learns from the rollout (examples/sequence_policy.py)."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


def _policy(dtype, sims=24, dim=64, hidden=96, actions=6):
    from examples.sequence_policy import SequencePolicy
    return SequencePolicy(dim, hidden, actions, sims, dtype=dtype)


def _reference(p, x, done, h0):
    """The same block in 64 bits with torch's own derivatives."""
    def norm(s, g, b):
        mean = s.mean(-1, keepdim=True)
        return (s - mean) / torch.sqrt(((s - mean) ** 2).mean(-1, keepdim=True) + 1e-5) * g + b

    n1 = norm(x, p["g1"], p["b1"])
    f, v = n1 @ p["w_f"].T, n1 @ p["w_v"].T
    c, out = h0, []
    for t in range(x.shape[0]):
        a = torch.sigmoid(f[t])
        h = a * c + (1 - a) * v[t]
        out.append(h)
        c = torch.where(done[t][:, None], 0.0, h)
    s2 = x + torch.stack(out)
    n2 = norm(s2, p["g2"], p["b2"])
    g, u = n2 @ p["w_gate"].T, n2 @ p["w_up"].T
    s3 = s2 + (g * torch.sigmoid(g) * u) @ p["w_down"].T
    return norm(s3, p["g3"], p["b3"]) @ p["w_head"].T


def test_acting_and_learning_agree_with_the_definition():
    """float16: every stored intermediate is rounded to 2^-11 of itself, some ten of them one after another; values within
    2 %, gradients (twice as many) within 4 % in the 2-norm."""
    sims, steps, dim, actions = 24, 7, 64, 6
    policy = _policy(torch.float16)
    gen = torch.Generator().manual_seed(3)
    x = torch.randn(steps, sims, dim, generator=gen).half().cuda()
    done = (torch.rand(steps, sims, generator=gen) < 0.2).cuda()
    adv = torch.randn(steps, sims, generator=gen).cuda()
    u = torch.rand(steps, sims, generator=gen).cuda()
    policy.memory.copy_(torch.randn(sims, dim, generator=gen))
    h0 = policy.memory.clone()
    p64 = {k: v.double().requires_grad_() for k, v in policy.p.items()}
    want = _reference(p64, x.double(), done, h0.double())
    # acting, one step at a time with the memory in place
    acts, logps = zip(*(policy.act(x[t], u[t], done[t]) for t in range(steps)))
    acts, logps = torch.stack(acts), torch.stack(logps)
    dist = torch.log_softmax(want, -1)
    chosen = dist.gather(-1, acts.unsqueeze(-1).long())[..., 0]
    assert float((logps.double() - chosen).abs().max()) < 0.02 * float(dist.abs().max())
    # learning from the rollout
    loss, grads, logits = policy.learn(x, acts, adv, done, h0)
    assert float((logits.double().view_as(want) - want).norm() / want.norm()) < 0.02
    want_loss = -(chosen * adv.double()).mean()
    want_loss.backward()
    assert abs(float(loss) - float(want_loss)) < 0.02 * float((chosen * adv.double()).abs().mean())
    for k, v in p64.items():
        rel = float((grads[k].double() - v.grad).norm() / v.grad.norm())
        assert rel < 0.04, (k, rel)


def test_the_example_learns_what_needs_the_memory():
    """The rewarded action is the previous step's cue: without the memory no policy passes 1/4."""
    from examples.sequence_policy import main
    rates = main(["--sims", "512", "--rounds", "60"])
    assert sum(rates[-5:]) / 5 > 0.5, rates[-5:]
