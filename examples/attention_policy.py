"""A small policy that remembers by attention, built from the operators of paper_1906_04585_b200.sequence, acting and learning.

One pre-norm block over the steps of a rollout, in which episodes end and begin anew:

    n1 = layer_norm(x)        q, k, v = heads of n1 W^T          q, k = qk_norm_rotary(q, k) at the step of the episode
    s2 = x + linear_attention(q, k, v) Wo^T                      n2 = layer_norm(s2)
    s3 = s2 + gated_ffn(n2)   n3 = layer_norm(s3)                logits = adjust_logits(n3 Wh^T, the actions allowed)

Acting takes one step at a time: the memory of every simulator, one matrix a head, is kept in place between calls, an episode's
end empties it, and the action is drawn by `sample` from the actions that the state allows.  Learning takes the whole rollout at
once and returns the gradients of a policy gradient loss, mean over steps of -advantage * log pi(action).

    python examples/attention_policy.py [--sims 64 --steps 5 --rounds 20]

runs rounds of both on a task that needs the memory (the rewarded action is the cue shown one step earlier).
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_1906_04585_b200 import sequence as S  # noqa: E402


class AttentionPolicy:
    def __init__(self, dim, heads, hidden, actions, sims, seed=1, dtype=torch.bfloat16):
        gen = torch.Generator().manual_seed(seed)
        self.heads, self.width = heads, dim // heads

        def mat(n, m):
            return (torch.randn(n, m, generator=gen) * m ** -0.5).to(dtype).cuda()

        self.p = {"w_qkv": mat(3 * dim, dim), "w_o": mat(dim, dim), "w_gate": mat(hidden, dim), "w_up": mat(hidden, dim), "w_down": mat(dim, hidden),
                  "w_head": mat(actions, dim)}
        for k in ("1", "2", "3"):
            self.p["g" + k], self.p["b" + k] = torch.ones(dim, dtype=dtype, device="cuda"), torch.zeros(dim, dtype=dtype, device="cuda")
        for k in ("gq", "gk"):
            self.p[k] = torch.ones(self.width, dtype=dtype, device="cuda")
        # heads that remember for 2 to 64 steps
        self.log_decay = torch.log1p(-torch.exp2(-torch.linspace(1.0, 6.0, heads, dtype=torch.float64))).float().cuda()
        self.inv_freq = torch.pow(10000.0, -torch.arange(self.width // 2, dtype=torch.float64) * 2 / self.width).float().cuda()
        self.memory = torch.zeros(sims, heads, self.width, self.width, device="cuda")
        self.position = torch.zeros(sims, dtype=torch.int32, device="cuda")

    def _forward(self, x, positions, allowed, s0, done, s_last, save):
        """x [steps, sims, dim]; positions and done [steps, sims]; allowed: bit masks [steps * sims, words] or None.  Returns the
        logits and what the backward pass needs."""
        p, (T, N, D) = self.p, x.shape
        H, W = self.heads, self.width
        s1 = x.reshape(T * N, D)
        n1, _, mean1, rstd1 = S.layer_norm(s1, p["g1"], p["b1"])
        q0, k0, v = (n1 @ p["w_qkv"].T).view(T * N, 3, H, W).unbind(1)
        at = positions.reshape(-1)
        q, k = S.qk_norm_rotary(q0, k0, at, self.inv_freq, p["gq"], p["gk"])
        q4, k4, v4 = q.view(T, N, H, W), k.view(T, N, H, W), v.unflatten(0, (T, N))
        o, _ = S.linear_attention(q4, k4, v4, self.log_decay, s0, done=done, s_last=s_last)
        o = o.view(T * N, D)
        n2, s2, mean2, rstd2 = S.layer_norm(s1, p["g2"], p["b2"], residual=o @ p["w_o"].T)
        y, saved = S.gated_ffn(n2, p["w_gate"], p["w_up"], p["w_down"], save=save)
        n3, s3, mean3, rstd3 = S.layer_norm(s2, p["g3"], p["b3"], residual=y)
        logits = n3 @ p["w_head"].T
        if allowed is not None:
            logits = S.adjust_logits(logits, mask=allowed, out=logits)
        return logits, (s1, n1, mean1, rstd1, q0, k0, at, q4, k4, v4, o, n2, s2, mean2, rstd2, saved, n3, s3, mean3, rstd3)

    def act(self, x, uniforms, allowed=None, done=None):
        """One step for all simulators, x [sims, dim]; done: whose episode ends with this step.  (actions, logprobs)"""
        logits, _ = self._forward(x.unsqueeze(0), self.position.unsqueeze(0), allowed, self.memory, None if done is None else done.unsqueeze(0), self.memory, False)
        self.position += 1
        if done is not None:
            self.position[done] = 0
        return S.sample(logits, uniforms)

    def learn(self, x, positions, actions, advantages, done, s0, allowed=None):
        """Gradients of the loss over a rollout, x [steps, sims, dim], positions, actions, advantages and done [steps, sims];
        s0: the memory before it.  (loss, {parameter: gradient}, logits)"""
        p, (T, N, D) = self.p, x.shape
        logits, (s1, n1, mean1, rstd1, q0, k0, at, q, k, v, o, n2, s2, mean2, rstd2, saved, n3, s3, mean3, rstd3) = self._forward(
            x, positions, allowed, s0, done, torch.empty_like(s0), True)
        taken = actions.reshape(-1, 1).long()
        adv = advantages.reshape(-1)
        logp = torch.log_softmax(logits.float(), 1)
        dlogits = logp.exp()
        dlogits.scatter_add_(1, taken, torch.full_like(dlogits[:, :1], -1.0))
        dlogits = (dlogits * (adv / (T * N)).unsqueeze(1)).to(x.dtype)
        g = {"w_head": dlogits.T @ n3}
        ds3, g["g3"], g["b3"] = S.layer_norm_backward(dlogits @ p["w_head"], s3, mean3, rstd3, p["g3"])
        dn2, g["w_gate"], g["w_up"], g["w_down"] = S.gated_ffn_backward(ds3, n2, p["w_gate"], p["w_up"], p["w_down"], saved)
        ds2, g["g2"], g["b2"] = S.layer_norm_backward(dn2, s2, mean2, rstd2, p["g2"], dsum=ds3)
        g["w_o"] = ds2.T @ o
        dqkv = torch.empty(T * N, 3, self.heads, self.width, dtype=x.dtype, device=x.device)
        dq, dk, dv, _ = S.linear_attention_backward((ds2 @ p["w_o"]).view_as(v), q, k, v, self.log_decay, s0, done=done, dv=dqkv[:, 2].unflatten(0, (T, N)))
        _, _, g["gq"], g["gk"] = S.qk_norm_rotary_backward(dq.flatten(0, 1), dk.flatten(0, 1), q0, k0, at, self.inv_freq, p["gq"], p["gk"], dq=dqkv[:, 0],
                                                           dk=dqkv[:, 1])
        dqkv = dqkv.view(T * N, 3 * D)
        g["w_qkv"] = dqkv.T @ n1
        _, g["g1"], g["b1"] = S.layer_norm_backward(dqkv @ p["w_qkv"], s1, mean1, rstd1, p["g1"], dsum=ds2)
        return -(logp.gather(1, taken)[:, 0] * adv).mean(), g, logits


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--sims", type=int, default=1024)
    ap.add_argument("--steps", type=int, default=5)
    ap.add_argument("--rounds", type=int, default=60)
    ap.add_argument("--lr", type=float, default=0.5)
    a = ap.parse_args(argv)
    dim, actions = 128, 4
    gen = torch.Generator(device="cuda").manual_seed(7)
    policy = AttentionPolicy(dim, 4, 256, actions + 2, a.sims)      # two actions more than the states allow
    allowed = torch.full((a.sims, 1), (1 << actions) - 1, dtype=torch.int32, device="cuda")
    master = {k: v.float() for k, v in policy.p.items()}
    table = torch.randn(actions, dim, device="cuda", generator=gen).bfloat16()
    cue = torch.randint(0, actions, (a.sims,), device="cuda", generator=gen)
    rates = []
    for r in range(a.rounds):
        s0 = policy.memory.clone()
        obs, acts, rewards, dones, positions = [], [], [], [], []
        for t in range(a.steps):
            before, cue = cue, torch.randint(0, actions, (a.sims,), device="cuda", generator=gen)
            x = table[cue]
            done = torch.rand(a.sims, device="cuda", generator=gen) < 0.02
            positions.append(policy.position.clone())
            action, _ = policy.act(x, torch.rand(a.sims, device="cuda", generator=gen), allowed, done)
            obs.append(x), acts.append(action), dones.append(done), rewards.append((action == before).float())
        reward = torch.stack(rewards)
        loss, grads, _ = policy.learn(torch.stack(obs), torch.stack(positions), torch.stack(acts), reward - reward.mean(), torch.stack(dones), s0,
                                      allowed.repeat(a.steps, 1))
        for k, g in grads.items():
            master[k] -= a.lr * g.float()
            policy.p[k].copy_(master[k])
        rates.append(float(reward.mean()))
        if r % 10 == 0 or r == a.rounds - 1:
            print("round %3d  reward %.3f  (chance %.3f)" % (r, rates[-1], 1.0 / actions))
    S.check()
    return rates


if __name__ == "__main__":
    main()
