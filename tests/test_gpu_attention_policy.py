"""GPU: the operators of attention together - a policy that acts step by step and learns from the rollout
(examples/attention_policy.py)."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


def _reference(policy, p, x, positions, allowed, done, s0):
    """The same block in 64 bits with torch's own derivatives."""
    T, N, D = x.shape
    H, W = policy.heads, policy.width

    def norm(s, g, b):
        mean = s.mean(-1, keepdim=True)
        return (s - mean) / torch.sqrt(((s - mean) ** 2).mean(-1, keepdim=True) + 1e-5) * g + b

    def turned(y, w):
        y = y / torch.sqrt(y.pow(2).mean(-1, keepdim=True) + 1e-6) * w
        f = positions.double().unsqueeze(-1) * policy.inv_freq.double()
        c, s = torch.cos(f).unsqueeze(2), torch.sin(f).unsqueeze(2)
        a, b = y.chunk(2, -1)
        return torch.cat([a * c - b * s, b * c + a * s], -1)

    n1 = norm(x, p["g1"], p["b1"])
    q, k, v = (n1 @ p["w_qkv"].T).view(T, N, 3, H, W).unbind(2)
    q, k = turned(q, p["gq"]), turned(k, p["gk"])
    decay = torch.exp(policy.log_decay.double()).view(1, H, 1, 1)
    state, out = s0, []
    for t in range(T):
        state = decay * state + k[t].unsqueeze(-1) * v[t].unsqueeze(-2)
        out.append((q[t].unsqueeze(-2) @ state).squeeze(-2) * W ** -0.5)
        state = torch.where(done[t].view(-1, 1, 1, 1), 0.0, state)
    s2 = x + torch.stack(out).reshape(T, N, D) @ p["w_o"].T
    n2 = norm(s2, p["g2"], p["b2"])
    g, u = n2 @ p["w_gate"].T, n2 @ p["w_up"].T
    s3 = s2 + (g * torch.sigmoid(g) * u) @ p["w_down"].T
    logits = norm(s3, p["g3"], p["b3"]) @ p["w_head"].T
    at = torch.arange(logits.shape[-1], device=x.device)
    open_ = ((allowed[:, at // 32] >> (at % 32)) & 1 != 0).view_as(logits)
    return torch.where(open_, logits, -float("inf"))


@pytest.mark.parametrize("steps", [7, 150])
def test_acting_and_learning_agree_with_the_definition(steps):
    """float16: every stored intermediate is rounded to 2^-11 of itself, some fifteen of them one after another; values within
    3 %, gradients (twice as many) within 5 % in the 2-norm.  7 steps go through the memory at once, 150 by chunks."""
    from examples.attention_policy import AttentionPolicy
    sims, dim, heads, actions = 12, 64, 2, 6
    policy = AttentionPolicy(dim, heads, 96, actions, sims, dtype=torch.float16)
    gen = torch.Generator().manual_seed(3)
    x = torch.randn(steps, sims, dim, generator=gen).half().cuda()
    done = (torch.rand(steps, sims, generator=gen) < 0.1).cuda()
    adv = torch.randn(steps, sims, generator=gen).cuda()
    u = torch.rand(steps, sims, generator=gen).cuda()
    allowed = (torch.randint(0, 1 << actions, (steps * sims, 1), generator=gen) | 1 | 1 << 4).to(torch.int32).cuda()
    policy.memory.copy_(torch.randn(sims, heads, dim // heads, dim // heads, generator=gen))
    s0 = policy.memory.clone()
    acts, logps, positions = [], [], []
    for t in range(steps):
        positions.append(policy.position.clone())
        a, l = policy.act(x[t], u[t], allowed[t * sims:(t + 1) * sims], done[t])
        acts.append(a), logps.append(l)
    acts, logps, positions = torch.stack(acts), torch.stack(logps), torch.stack(positions)
    p64 = {k: v.double().requires_grad_() for k, v in policy.p.items()}
    want = _reference(policy, p64, x.double(), positions, allowed, done, s0.double())
    dist = torch.log_softmax(want, -1)
    chosen = dist.gather(-1, acts.unsqueeze(-1).long())[..., 0]
    assert torch.isfinite(chosen).all()
    scale = float(dist[torch.isfinite(dist)].abs().max())
    assert float((logps.double() - chosen).abs().max()) < 0.03 * scale
    loss, grads, logits = policy.learn(x, positions, acts, adv, done, s0, allowed)
    got, fine = logits.double().view_as(want), torch.isfinite(want)
    assert torch.equal(fine, torch.isfinite(got))
    assert float((got - want)[fine].norm() / want[fine].norm()) < 0.03
    want_loss = -(chosen * adv.double()).mean()
    want_loss.backward()
    assert abs(float(loss) - float(want_loss)) < 0.03 * float((chosen * adv.double()).abs().mean())
    for k, v in p64.items():
        rel = float((grads[k].double() - v.grad).norm() / v.grad.norm())
        assert rel < 0.05, (k, rel)


def test_the_example_runs():
    from examples.attention_policy import main
    rates = main(["--sims", "128", "--rounds", "3"])
    assert len(rates) == 3 and all(0.0 <= r <= 1.0 for r in rates)
