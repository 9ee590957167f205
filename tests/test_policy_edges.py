"""The policy loss where a term is switched off or leaves fp32's range."""
import pytest
import torch

import paper_1907_12205_b200 as dx

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TYPES = [torch.bfloat16, torch.float16, torch.float32]
INF = float("inf")


def rows_of(n, vocab, dtype, seed=0):
    gen = torch.Generator(device=DEV).manual_seed(seed)
    return (2 * torch.randn((n, vocab), generator=gen, device=DEV)).to(dtype), torch.randint(0, vocab, (n,), generator=gen, device=DEV)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("vocab", [40, 3001, 40000])
def test_a_kl_term_without_weight_counts_nowhere_but_in_its_statistic(dtype, vocab):
    n = 7
    z, y = rows_of(n, vocab, dtype)
    z[5, y[5]] = -INF                              # a chosen token that the policy gives nothing: the gap is infinite
    logp = torch.log_softmax(z.double(), 1).gather(1, y[:, None])[:, 0]
    old = torch.where(logp.isinf(), -3.0, logp + 0.1).float()
    ref = torch.where(logp.isinf(), -4.0, logp).float() + torch.tensor([0.0, 60.0, 88.0, 100.0, 700.0, 1.0, INF], device=DEV)
    a = torch.tensor([1.0, -1.0, 0.5, 2.0, -0.3, 1.0, 0.7], device=DEV)
    w = torch.full((n,), 0.125, device=DEV)
    plain = dx.detox_policy_loss(z, y, old, a, None, w, kl_coef=0.0)
    got = dx.detox_policy_loss(z, y, old, a, ref, w, kl_coef=0.0)
    assert bool(got.stats[:2].isfinite().all()) and bool(got.dz.isfinite().all())
    assert torch.equal(got.stats[[0, 1, 3]], plain.stats[[0, 1, 3]]) and torch.equal(got.dz, plain.dz) and torch.equal(got.logp, plain.logp)
    assert float(got.kl) == INF and float(plain.kl) == 0.0
    # and where no row is that far the statistic is the sum
    near = dx.detox_policy_loss(z[:1], y[:1], old[:1], a[:1], old[:1], w[:1], kl_coef=0.0)
    d = old[:1].double() - logp[:1]
    assert abs(float(near.kl) - 0.125 * float(torch.expm1(d) - d)) <= 1e-6 * 0.125


@pytest.mark.parametrize("dtype", TYPES)
def test_a_ratio_beyond_the_range_with_an_advantage_of_zero(dtype):
    n = 5
    z, y = rows_of(n, 50, dtype)
    logp = torch.log_softmax(z.double(), 1).gather(1, y[:, None])[:, 0]
    old = (logp - torch.tensor([100.0, 700.0, 100.0, 0.1, 100.0], device=DEV)).float()
    a = torch.tensor([0.0, -0.0, 2.0, 1.0, 0.0], device=DEV)
    w = torch.full((n,), 0.25, device=DEV)
    got = dx.detox_policy_loss(z, y, old, a, None, w, clip_low=0.2, clip_high=0.3)
    # rows 0, 1 and 4 count nothing, row 2 is clipped at 1.3, row 3 is inside
    want = -0.25 * (1.3 * 2.0 + float(torch.exp(logp[3] - old[3].double())))
    assert abs(float(got.loss) - want) <= 1e-5 and abs(float(got.clipped) - 0.25) == 0.0
    assert bool((got.dz[[0, 1, 2, 4]] == 0).all()) and bool(got.dz.isfinite().all()) and bool((got.dz[3] != 0).any())
    # where it is infinite, or a number is missing, that shows
    bad = dx.detox_policy_loss(z[:1], y[:1], torch.tensor([-INF], device=DEV), a[:1], None, w[:1])
    assert bool(bad.loss.isnan())
    bad = dx.detox_policy_loss(z[:1], y[:1], torch.tensor([float("nan")], device=DEV), a[:1], None, w[:1])
    assert bool(bad.loss.isnan())
