"""A small policy with a memory, built from the operators of paper_1906_04585_b200.sequence, acting and learning.

One pre-norm residual block over the steps of a rollout:

    s1 = x                  n1 = layer_norm(s1)       f, v = n1 Wf^T, n1 Wv^T      m = gated_recurrence(f, v)
    s2 = s1 + m             n2 = layer_norm(s2)       y = gated_ffn(n2)
    s3 = s2 + y             n3 = layer_norm(s3)       logits = n3 Wh^T

Acting takes one step at a time: the memory of every simulator is kept in place between calls, an episode's end empties
it, and the action is drawn by `sample`.  Learning takes the whole rollout at once and returns the gradients of a policy
gradient loss, mean over steps of -advantage * log pi(action).  Plain projections are torch products.

    python examples/sequence_policy.py [--sims 64 --steps 5 --rounds 20]

runs rounds of both on a task that needs the memory (the rewarded action is the cue shown one step earlier).
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_1906_04585_b200 import sequence as S  # noqa: E402


class SequencePolicy:
    def __init__(self, dim, hidden, actions, sims, seed=1, dtype=torch.bfloat16):
        gen = torch.Generator().manual_seed(seed)

        def mat(n, m):
            return (torch.randn(n, m, generator=gen) * m ** -0.5).to(dtype).cuda()

        self.p = {"w_f": mat(dim, dim), "w_v": mat(dim, dim), "w_gate": mat(hidden, dim), "w_up": mat(hidden, dim), "w_down": mat(dim, hidden),
                  "w_head": mat(actions, dim)}
        for k in ("1", "2", "3"):
            self.p["g" + k], self.p["b" + k] = torch.ones(dim, dtype=dtype, device="cuda"), torch.zeros(dim, dtype=dtype, device="cuda")
        self.memory = torch.zeros(sims, dim, device="cuda")

    def _forward(self, x, h0, done, h_last, save):
        """x [steps, sims, dim]; returns the logits and what the backward pass needs."""
        p, (T, N, D) = self.p, x.shape
        s1 = x.reshape(T * N, D)
        n1, _, mean1, rstd1 = S.layer_norm(s1, p["g1"], p["b1"])
        f, v = (n1 @ p["w_f"].T).view(T, N, D), (n1 @ p["w_v"].T).view(T, N, D)
        m, _, states = S.gated_recurrence(f, v, h0, done=done, h_last=h_last, save=save)
        n2, s2, mean2, rstd2 = S.layer_norm(s1, p["g2"], p["b2"], residual=m.view(T * N, D))
        y, saved = S.gated_ffn(n2, p["w_gate"], p["w_up"], p["w_down"], save=save)
        n3, s3, mean3, rstd3 = S.layer_norm(s2, p["g3"], p["b3"], residual=y)
        return n3 @ p["w_head"].T, (s1, n1, mean1, rstd1, f, v, states, n2, s2, mean2, rstd2, saved, n3, s3, mean3, rstd3)

    def act(self, x, uniforms, done=None):
        """One step for all simulators, x [sims, dim]; done: whose episode ends with this step.  (actions, logprobs)"""
        logits, _ = self._forward(x.unsqueeze(0), self.memory, None if done is None else done.unsqueeze(0), self.memory, False)
        return S.sample(logits, uniforms)

    def learn(self, x, actions, advantages, done, h0):
        """Gradients of the loss over a rollout, x [steps, sims, dim], actions, advantages and done [steps, sims]; h0: the
        memory before it.  (loss, {parameter: gradient}, logits)"""
        p, (T, N, D) = self.p, x.shape
        h_last = torch.empty_like(h0)
        logits, (s1, n1, mean1, rstd1, f, v, states, n2, s2, mean2, rstd2, saved, n3, s3, mean3, rstd3) = self._forward(x, h0, done, h_last, True)
        logp = torch.log_softmax(logits.float(), 1)
        taken = logp.gather(1, actions.reshape(-1, 1).long())[:, 0]
        adv = advantages.reshape(-1)
        dlogits = torch.softmax(logits.float(), 1)
        dlogits.scatter_add_(1, actions.reshape(-1, 1).long(), torch.full_like(dlogits[:, :1], -1.0))
        dlogits = (dlogits * (adv / (T * N)).unsqueeze(1)).to(x.dtype)
        g = {"w_head": dlogits.T @ n3}
        ds3, g["g3"], g["b3"] = S.layer_norm_backward(dlogits @ p["w_head"], s3, mean3, rstd3, p["g3"])
        dn2, g["w_gate"], g["w_up"], g["w_down"] = S.gated_ffn_backward(ds3, n2, p["w_gate"], p["w_up"], p["w_down"], saved)
        ds2, g["g2"], g["b2"] = S.layer_norm_backward(dn2, s2, mean2, rstd2, p["g2"], dsum=ds3)
        df, dv, _ = S.gated_recurrence_backward(ds2.view(T, N, D), f, v, states, done=done)
        df, dv = df.view(T * N, D), dv.view(T * N, D)
        g["w_f"], g["w_v"] = df.T @ n1, dv.T @ n1
        _, g["g1"], g["b1"] = S.layer_norm_backward(df @ p["w_f"] + dv @ p["w_v"], s1, mean1, rstd1, p["g1"], dsum=ds2)
        return -(taken * adv).mean(), g, logits


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--sims", type=int, default=1024)
    ap.add_argument("--steps", type=int, default=5)
    ap.add_argument("--rounds", type=int, default=60)
    ap.add_argument("--lr", type=float, default=0.5)
    a = ap.parse_args(argv)
    dim, actions = 128, 4
    gen = torch.Generator(device="cuda").manual_seed(7)
    policy = SequencePolicy(dim, 256, actions, a.sims)
    master = {k: v.float() for k, v in policy.p.items()}
    table = torch.randn(actions, dim, device="cuda", generator=gen).bfloat16()
    cue = torch.randint(0, actions, (a.sims,), device="cuda", generator=gen)
    rates = []
    for r in range(a.rounds):
        h0 = policy.memory.clone()
        obs, acts, rewards, dones = [], [], [], []
        for t in range(a.steps):
            before, cue = cue, torch.randint(0, actions, (a.sims,), device="cuda", generator=gen)
            x = table[cue]
            done = torch.rand(a.sims, device="cuda", generator=gen) < 0.02
            action, _ = policy.act(x, torch.rand(a.sims, device="cuda", generator=gen), done)
            obs.append(x), acts.append(action), dones.append(done), rewards.append((action == before).float())
        reward = torch.stack(rewards)
        loss, grads, _ = policy.learn(torch.stack(obs), torch.stack(acts), reward - reward.mean(), torch.stack(dones), h0)
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
