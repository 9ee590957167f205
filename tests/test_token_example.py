"""The example of redundant workers over tokens: it runs, its honest copies agree bit for bit, and its gradients are those of the loss."""
import math
import os
import sys

import pytest
import torch

import paper_1907_12205_b200 as dx

pytestmark = pytest.mark.gpu
DEV = "cuda:0"

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


@pytest.mark.parametrize("tokens,vocab,dim,hidden", [(64, 40, 64, 176), (130, 101, 72, 201)])
def test_the_example_runs(tokens, vocab, dim, hidden):
    import token_workers as example
    rewards, equal = example.train(steps=4, tokens=tokens, vocab=vocab, dim=dim, hidden=hidden, log=None)
    assert equal and len(rewards) == 4 and all(math.isfinite(r) for r in rewards)


def test_its_gradient_is_the_loss_gradient():
    """Against the same loss in 64 bits.  Kept activations are off by up to 2^-4 of an entry (3.6 % rms), each of the two gated factors by one and each gradient behind them
    by both, and every product's rows by bf16's 2^-9: together less than 10 % of a gradient's norm."""
    import token_workers as example
    vocab, dim, hidden, n = 50, 64, 176, 200
    policy = example.Policy(vocab, dim, hidden, DEV)
    gen = torch.Generator(device=DEV).manual_seed(3)
    seen = torch.randint(0, vocab, (n,), generator=gen, device=DEV)
    chosen = torch.randint(0, vocab, (n,), generator=gen, device=DEV)
    chosen[::17] = -1
    z, _ = policy.forward(seen)
    logp = dx.detox_token_logp(z, chosen).logp
    old = logp + 0.05 * torch.randn(n, generator=gen, device=DEV)      # ratios inside the border
    advantage = torch.randn(n, generator=gen, device=DEV)
    reference = logp + 0.2 * torch.randn(n, generator=gen, device=DEV)
    row = torch.empty(policy.size, device=DEV)
    policy.gradient(seen, chosen, old, advantage, reference, row)

    w = {k: v.double().requires_grad_() for k, v in policy.w.items()}
    x = w["table"][seen] * math.sqrt(dim)
    y = x * torch.rsqrt(x.square().mean(1, keepdim=True) + example.EPS) * w["norm"]
    h = torch.nn.functional.silu(y @ w["gate"].T) * (y @ w["up"].T)
    logits = (x + h @ w["down"].T) @ w["table"].T
    new = torch.log_softmax(logits, 1).gather(1, chosen.clamp(min=0)[:, None])[:, 0]
    r = torch.exp(new - old.double())
    a = advantage.double()
    gap = reference.double() - new
    each = -torch.minimum(r * a, r.clamp(1 - example.LOW, 1 + example.HIGH) * a) + example.KL * (torch.exp(gap) - gap - 1)
    (torch.where(chosen >= 0, each, 0.0).sum() / n).backward()
    for name, g in policy.pieces(row).items():
        want = w[name].grad
        assert float((g.double() - want).norm() / want.norm()) < 0.1, name


def test_one_step_takes_the_gradient_into_the_weights():
    import token_workers as example
    policy = example.Policy(40, 64, 176, DEV)
    before, g = policy.flat.clone(), torch.randn(policy.size, device=DEV)
    policy.step(g, 1, 0.01)
    # the first step moves every entry by lr g / (|g| + eps), which is lr against its gradient's sign but for lr eps / |g| (some |g| are 10^-5 here: 10^-5 of
    # it), and by lr x 0.01 of itself at most
    moved = policy.flat - before
    assert bool(((moved + 0.01 * torch.sign(g)).abs() <= 1e-4 * before.abs() + 2e-6 + 0.01 * 1e-8 / g.abs()).all())
    for name, w in policy.pieces(policy.flat).items():
        assert torch.equal(policy.w[name], w.to(torch.bfloat16))
