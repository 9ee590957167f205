"""Redundant workers train a gated feed-forward sublayer; the server votes on their gradients.

n workers in groups of r compute the gradient of the sublayer

    s = x + residual,   y = rmsnorm(s),   h = silu(y Wg^T) * (y Wu^T),   out = s + h Wd^T

on their group's batch (Algorithm 1, lines 2-6: every member of a group works on the same files).  Between the forward and the
backward pass a worker keeps y, g and u in 8 bits.  The vote needs the honest copies of a gradient to be equal bit for bit, which
the operators' fixed order of additions gives; some workers are Byzantine and send the reversed gradient.  The server takes
the majority of each group, the mean over sets of votes and the median of those.

  python examples/feed_forward_workers.py [--steps 20] [--tokens 256] [--dim 256] [--hidden 704]
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


class Sublayer:
    """The weights in fp32, as slices of one vector (a gradient is a row of the same layout), and in bf16 for the products."""

    def __init__(self, dim: int, hidden: int, device: str):
        self.shapes = {"norm": (dim,), "gate": (hidden, dim), "up": (hidden, dim), "down": (dim, hidden)}
        self.size = sum(math.prod(s) for s in self.shapes.values())
        gen = torch.Generator(device=device).manual_seed(1)
        self.flat = torch.randn(self.size, generator=gen, device=device)
        w = self.pieces(self.flat)
        w["norm"].fill_(1.0)
        for name in ("gate", "up", "down"):
            w[name] /= math.sqrt(self.shapes[name][1])
        self.round()

    def pieces(self, row: torch.Tensor):
        out, at = {}, 0
        for name, shape in self.shapes.items():
            out[name] = row[at: at + math.prod(shape)].view(shape)
            at += math.prod(shape)
        return out

    def round(self):
        self.w = {k: v.to(torch.bfloat16) for k, v in self.pieces(self.flat).items()}

    def gradient(self, x: torch.Tensor, residual: torch.Tensor, target: torch.Tensor, row: torch.Tensor) -> torch.Tensor:
        """Writes the gradient of mean((out - target)^2) / 2 over the batch into `row`; returns the loss."""
        w, out = self.w, self.pieces(row)
        norm = dx.detox_rmsnorm(x, w["norm"], residual, eps=EPS, want_q=True)
        h, kept = dx.detox_gated(norm.y, w["gate"], w["up"], dx.ACT_SILU, keep=True)
        saved = (norm.q, norm.e)                                   # what stays until the backward pass: 8 bits an entry
        err = (norm.sum + h @ w["down"].T).float() - target
        loss = err.square().mean() / 2

        dout = (err / err.numel()).to(torch.bfloat16)
        out["down"].copy_((dout.T @ h).float())
        dh = dout @ w["down"]
        dy, _, _ = dx.detox_gated_backward(dh, saved, w["gate"], w["up"], dx.ACT_SILU, kept=kept, dwg=out["gate"], dwu=out["up"])
        dx.detox_rmsnorm_backward(dy, norm.sum, w["norm"], norm.rstd, ds=dout, dw=out["norm"])
        return loss


def train(steps: int = 20, tokens: int = 256, dim: int = 256, hidden: int = 704, n: int = 15, r: int = 3, byzantine: int = 3,
          lr: float = 40.0, device: str = "cuda:0", log=print):
    """Returns the mean loss of every step, and whether every group's honest rows were equal bit for bit."""
    layer = Sublayer(dim, hidden, device)
    rng = np.random.default_rng(0)
    gen = torch.Generator(device=device).manual_seed(2)
    teacher = Sublayer(dim, hidden, device).pieces(torch.randn(layer.size, generator=gen, device=device))
    groups = n // r
    ld = (layer.size + 31) // 32 * 32
    X = torch.zeros((n, ld), device=device)[:, : layer.size]       # the received gradients
    sets = [0, groups // 2, groups]
    losses, equal = [], True
    for step in range(steps):
        members = rng.permutation(n).astype(np.int32)
        losing = rng.choice(groups, byzantine, replace=False)      # one attacker in each of these groups
        total = 0.0
        for j in range(groups):
            x, residual = (torch.randn((tokens, dim), generator=gen, device=device).to(torch.bfloat16) for _ in range(2))
            s = (x + residual).float()
            y = s * torch.rsqrt(s.square().mean(1, keepdim=True) + EPS)
            target = s + torch.tanh(y @ teacher["gate"].T / math.sqrt(dim)) @ teacher["down"].T / math.sqrt(hidden)
            own = members[j * r: (j + 1) * r]
            for worker in own:                                     # every member computes it for itself
                loss = layer.gradient(x, residual, target, X[worker])
            equal = equal and all(torch.equal(X[own[0]].view(torch.int32), X[k].view(torch.int32)) for k in own[1:])
            total += float(loss)
            if j in losing:
                X[own[step % r]] *= -100.0
        expired, first = dx.gated_expired_waits()                  # (a product that gave up has left NaN in its worker's row)
        if expired:
            raise RuntimeError(f"{expired} waits of the gated products ran out, the first: {first}")
        pipe = dx.Pipeline(n, r, layer.size, members, dx.AGG_MEAN, sets, np.arange(groups), dx.AGG_COORD_MEDIAN)
        res = dx.detox_aggregate(pipe, X)
        assert bool((res["winner"] >= 0).all()), "a group without a majority"
        layer.flat -= lr * res["out"]
        layer.round()
        losses.append(total / groups)
        if log:
            log(f"step {step:3d}  loss {losses[-1]:.4f}")
    return losses, equal


def main():
    p = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    for name, value in (("steps", 20), ("tokens", 256), ("dim", 256), ("hidden", 704)):
        p.add_argument(f"--{name}", type=int, default=value)
    a = p.parse_args()
    losses, equal = train(a.steps, a.tokens, a.dim, a.hidden)
    print("honest copies of every gradient equal bit for bit:", equal)


if __name__ == "__main__":
    main()
