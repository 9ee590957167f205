"""Entries masked by finite numbers of any size, beside a chosen token that is among them or not."""
import pytest
import torch

import paper_1907_12205_b200 as dx

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
U = 2.0 ** -24


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("mask", [-1e4, -1e9, -1e10, -1e20, -3e26, -1e28, -1e30, -3e38])
@pytest.mark.parametrize("scale", [0.7, 1.0, 1.3])
@pytest.mark.parametrize("vocab", [2, 40, 3001, 40000])
def test_masked_by_a_finite_number(dtype, mask, scale, vocab):
    """Row 0: the chosen token alone is left.  Row 1: it and another (or it alone).  Row 2: it is masked itself, another is left.  Row 3: nothing is masked."""
    gen = torch.Generator(device=DEV).manual_seed(vocab)
    z = torch.randn((4, vocab), generator=gen, device=DEV)
    y = torch.tensor([0, vocab - 1, 1, 0], device=DEV)
    keep = torch.zeros((4, vocab), dtype=torch.bool, device=DEV)
    keep[0, 0] = keep[1, vocab - 1] = keep[1, vocab // 3] = keep[2, 0] = True
    keep[3] = True
    z = torch.where(keep, z, torch.tensor(mask, device=DEV)).to(dtype)
    scale = float(torch.tensor(scale))
    x = z.double() * scale
    exact = torch.log_softmax(x, 1)
    logp = exact.gather(1, y[:, None])[:, 0]
    got = dx.detox_token_logp(z, y, scale=scale)
    fine = torch.tensor([True, True, False, True], device=DEV)
    off = 400 * U
    old = torch.where(fine, logp + 0.05, -2.0).float()
    one, w = torch.ones(4, device=DEV), torch.full((4,), 0.25, device=DEV)
    pol = dx.detox_policy_loss(z, y, old, one, old, w, kl_coef=0.0, scale=scale)
    pairs = dx.detox_preference_loss(z[[0, 1, 3, 3]], y[[0, 1, 3, 3]], torch.tensor([0, 2, 4], dtype=torch.int32, device=DEV), torch.zeros(2, device=DEV), scale=scale)
    for one_of in (got.logp, pol.logp):
        assert bool(((one_of.double() - logp).abs() <= off)[fine].all())
        assert float(one_of[2]) <= 0.9 * float(logp[2])                  # or -Inf, where it counts as nothing
    assert bool(((got.lse.double() - torch.logsumexp(x, 1)).abs() <= off).all())
    assert bool(pol.stats[:2].isfinite().all()) and bool(pol.dz.isfinite().all()) and bool(pairs.dz.isfinite().all()) and bool(pairs.loss.isfinite().all())
    ratio = torch.where(fine, torch.exp(logp - old.double()), 0.0)
    assert abs(float(pol.loss) + 0.25 * float(ratio.clamp(max=1.2).sum())) <= 4 * off
    # the gradient: -ratio / 4 (1[j = y] - p_j) scale, nothing of a row whose ratio is nothing
    own = torch.zeros_like(exact).scatter_(1, y[:, None], 1.0)
    want = -0.25 * scale * ratio[:, None] * (own - torch.exp(exact))
    half = torch.finfo(dtype).eps / 2
    assert bool(((pol.dz.double() - want).abs() <= want.abs() * (half * 1.01 + 400 * U) + 0.25 * scale * off * torch.exp(exact) + 2.0 ** -126).all())


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("vocab", [1, 40, 3001, 40000])
def test_rows_masked_throughout(dtype, vocab):
    """By a number that fp32 still resolves: every entry alike.  By a larger one: empty."""
    y = torch.tensor([0, vocab - 1, vocab // 2], device=DEV)
    one = torch.ones(3, device=DEV)
    for mask, alike in ((-1e4, True), (-1e9, True), (1e9, True), (-1e10, False), (-1e20, False), (-1e30, False), (-3e38, False)):
        z = torch.full((3, vocab), mask, device=DEV).to(dtype)
        got, pol = dx.detox_token_logp(z, y), dx.detox_policy_loss(z, y, 0 * one, one, None, one, clip_low=1.0)
        logp = torch.log_softmax(z.double(), 1)[:, 0]
        if alike:
            for x in (got.logp, pol.logp):
                assert bool(((x.double() - logp).abs() <= 200 * U).all())
            assert bool(((got.lse.double() - torch.logsumexp(z.double(), 1)).abs() <= U * abs(mask) * 1.01 + 200 * U).all())
            assert bool(pol.dz.isfinite().all()) and (vocab == 1 or bool((pol.dz != 0).all()))
        else:
            assert bool((got.logp == float("-inf")).all()) and bool((got.lse == float("-inf")).all()) and bool((pol.logp == float("-inf")).all())
            assert bool((pol.dz == 0).all()) and float(pol.loss) == 0.0
