"""Redundant workers train a small policy over tokens; the server votes on their gradients and takes the result into the weights.

The policy: a token's row of a table, a pre-norm gated feed-forward sublayer, and the table again as output head,

    x = E[tokens],   out = x + gated(rmsnorm(x)) Wd^T,   logits = out E^T

Chosen tokens are rewarded when they follow a rule.  n workers in groups of r compute the gradient of the clipped policy loss with a KL term to the first policy, on
their group's batch and all from kernels that add in a fixed order, so that honest copies are equal bit for bit; some workers are
Byzantine.  The server takes the majority of each group, the mean over sets of votes and the median of those, and one AdamW step over all
tensors with states in 8 bits.

  python examples/token_workers.py [--steps 30] [--tokens 256] [--vocab 64] [--dim 64] [--hidden 176]
"""
from __future__ import annotations

import argparse
import math
import os
import sys

import numpy as np
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)

import paper_1907_12205_b200 as dx  # noqa: E402

EPS = 1e-6
LOW, HIGH, KL = 0.2, 0.2, 0.01


class Policy:
    """The weights in fp32, as slices of one vector (a gradient is a row of the same layout), and in bf16 for the products."""

    def __init__(self, vocab: int, dim: int, hidden: int, device: str):
        self.vocab = vocab
        self.shapes = {"table": (vocab, dim), "norm": (dim,), "gate": (hidden, dim), "up": (hidden, dim), "down": (dim, hidden)}
        self.size = sum(math.prod(s) for s in self.shapes.values())
        gen = torch.Generator(device=device).manual_seed(1)
        self.flat = torch.randn(self.size, generator=gen, device=device)
        w = self.pieces(self.flat)
        w["norm"].fill_(1.0)
        for name in ("table", "gate", "up", "down"):
            w[name] /= math.sqrt(self.shapes[name][1])
        self.w = {k: v.to(torch.bfloat16) for k, v in w.items()}
        self.m, self.v = dx.detox_adamw_state(list(self.w.values()), bits=8)

    def pieces(self, row: torch.Tensor):
        out, at = {}, 0
        for name, shape in self.shapes.items():
            out[name] = row[at: at + math.prod(shape)].view(shape)
            at += math.prod(shape)
        return out

    def forward(self, tokens: torch.Tensor):
        """(logits, what the backward pass needs)."""
        w = self.w
        x = dx.detox_embedding(tokens, w["table"], scale=math.sqrt(self.shapes["norm"][0]))
        norm = dx.detox_rmsnorm(x, w["norm"], eps=EPS, want_q=True)
        h, kept = dx.detox_gated(norm.y, w["gate"], w["up"], dx.ACT_SILU, keep=True)
        out = x + h @ w["down"].T
        return out @ w["table"].T, (x, norm, h, kept, out)

    def gradient(self, tokens, chosen, old, advantage, reference, row: torch.Tensor) -> dx.PolicyLoss:
        """Writes the gradient of the policy loss over the batch into `row`."""
        w, to = self.w, self.pieces(row)
        z, (x, norm, h, kept, out) = self.forward(tokens)
        loss = dx.detox_policy_loss(z, chosen, old, advantage, reference, clip_low=LOW, clip_high=HIGH, kl_coef=KL, dz=z)
        dz = loss.dz
        to["table"].copy_((dz.T @ out).float())                    # as output head; as embedding it comes on top below
        dout = dz @ w["table"]
        to["down"].copy_((dout.T @ h).float())
        dy, _, _ = dx.detox_gated_backward(dout @ w["down"], (norm.q, norm.e), w["gate"], w["up"], dx.ACT_SILU, kept=kept, dwg=to["gate"], dwu=to["up"])
        dx_, _ = dx.detox_rmsnorm_backward(dy, x, w["norm"], norm.rstd, ds=dout, dw=to["norm"])
        dx.detox_embedding_backward(dx_, tokens, self.vocab, scale=math.sqrt(self.shapes["norm"][0]), dw=to["table"], accumulate=True)
        return loss

    def step(self, gradient: torch.Tensor, number: int, lr: float):
        """One AdamW step along the aggregated gradient; the table and the norm's weight do not decay."""
        names = list(self.shapes)
        grads, masters = self.pieces(gradient), self.pieces(self.flat)
        dx.detox_adamw([self.w[n] for n in names], [grads[n] for n in names], self.m, self.v, number, lr, beta2=0.99,
                       weight_decay=[0.0 if n in ("table", "norm") else 0.01 for n in names], masters=[masters[n] for n in names], seed=7)


def train(steps: int = 30, tokens: int = 256, vocab: int = 64, dim: int = 64, hidden: int = 176, n: int = 15, r: int = 3, byzantine: int = 3,
          lr: float = 0.01, device: str = "cuda:0", log=print):
    """Returns the mean reward of every step, and whether every group's honest rows were equal bit for bit."""
    policy, first = Policy(vocab, dim, hidden, device), Policy(vocab, dim, hidden, device)
    rng = np.random.default_rng(0)
    gen = torch.Generator(device=device).manual_seed(2)
    groups = n // r
    X = torch.zeros((n, (policy.size + 31) // 32 * 32), device=device)[:, : policy.size]   # the received gradients
    sets = [0, groups // 2, groups]
    rewards, equal = [], True
    for step in range(1, steps + 1):
        members = rng.permutation(n).astype(np.int32)
        losing = rng.choice(groups, byzantine, replace=False)      # one attacker in each of these groups
        total = 0.0
        for j in range(groups):
            seen = torch.randint(0, vocab, (tokens,), generator=gen, device=device, dtype=torch.int32)
            seen[tokens - 3:] = -1                                 # padding: no token chosen there
            z, _ = policy.forward(seen)
            chosen = torch.multinomial(torch.softmax(z.float(), 1), 1, generator=gen)[:, 0].int()
            chosen[seen < 0] = -1
            old = dx.detox_token_logp(z, chosen, want_lse=False).logp
            reference = dx.detox_token_logp(first.forward(seen)[0], chosen, want_lse=False).logp
            reward = (chosen == (seen * 5 + 3) % vocab).float() * (seen >= 0)
            own = members[j * r: (j + 1) * r]
            for worker in own:                                     # every member computes it for itself
                policy.gradient(seen, chosen, old, reward - reward.mean(), reference, X[worker])
            equal = equal and all(torch.equal(X[own[0]].view(torch.int32), X[k].view(torch.int32)) for k in own[1:])
            total += float(reward.sum()) / (tokens - 3)
            if j in losing:
                X[own[step % r]] *= -100.0
        expired, what = dx.gated_expired_waits()                   # (a product that gave up has left NaN in its worker's row)
        if expired:
            raise RuntimeError(f"{expired} waits of the gated products ran out, the first: {what}")
        pipe = dx.Pipeline(n, r, policy.size, members, dx.AGG_MEAN, sets, np.arange(groups), dx.AGG_COORD_MEDIAN)
        res = dx.detox_aggregate(pipe, X)
        assert bool((res["winner"] >= 0).all()), "a group without a majority"
        policy.step(res["out"], step, lr)
        rewards.append(total / groups)
        if log:
            log(f"step {step:3d}  mean reward {rewards[-1]:.4f}")
    return rewards, equal


def main():
    p = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    for name, value in (("steps", 30), ("tokens", 256), ("vocab", 64), ("dim", 64), ("hidden", 176)):
        p.add_argument(f"--{name}", type=int, default=value)
    a = p.parse_args()
    _, equal = train(a.steps, a.tokens, a.vocab, a.dim, a.hidden)
    print("honest copies of every gradient equal bit for bit:", equal)


if __name__ == "__main__":
    main()
