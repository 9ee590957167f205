"""The temperature is taken to more than fp32's bits: an error of its would go the same way for every token of a sequence, and grow with the logits."""
import pytest
import torch

import paper_1907_12205_b200 as dx

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TYPES = [torch.bfloat16, torch.float16, torch.float32]
U = 2.0 ** -24
SCALES = [1.0, 0.7, 1.3, 1.5, 1 / 0.9]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("scale", SCALES)
def test_the_sums_of_long_sequences(dtype, scale):
    """One sequence of unlikely tokens and one of the likeliest.  Each power is known to 2^-22, its error's mean over entries to 3e-8 (the instruction's mean shortfall is put
    right), and nothing else has a mean: 6e-8 a token, and the sums' rounding to fp32 in the margin."""
    n, vocab, beta = 4000, 500, 0.5
    gen = torch.Generator(device=DEV).manual_seed(int(100 * scale))
    z = (12 * torch.randn((2 * n, vocab), generator=gen, device=DEV)).to(dtype)
    y = torch.cat([torch.randint(0, vocab, (n,), generator=gen, device=DEV), z[n:].argmax(1)])
    scale32 = float(torch.tensor(scale))
    logp = torch.log_softmax(z.double() * scale32, 1).gather(1, y[:, None])[:, 0]
    sums = torch.stack([logp[:n].sum(), logp[n:].sum()])
    ref = sums.float()
    got = dx.detox_preference_loss(z, y, torch.tensor([0, n, 2 * n], dtype=torch.int32, device=DEV), ref, beta=beta, scale=scale32, want_grad=False)
    gap = sums - ref.double()
    want = beta * float(gap[0] - gap[1])
    assert abs(float(got.margin[0]) - want) <= beta * 2 * n * 6e-8 + 2 * U * abs(want)
    assert bool(((got.sums.double() - sums).abs() <= U * sums.abs() + n * 6e-8).all())


@pytest.mark.parametrize("seed", [1, 2, 3])
def test_the_errors_of_powers_do_not_line_up(seed):
    """bf16 logits are multiples of one step where they count, so the same arguments come up in every row.  A power's error has a mean within 1e-8 of what is put right; over some
    twenty arguments that carry most of a sum it deviates by 1.4e-7 / sqrt(3) / sqrt(20) = 1.8e-8: two of those a token, and the margin's rounding."""
    n, vocab, beta, scale = 2000, 32000, 0.5, 1.25
    gen = torch.Generator(device=DEV).manual_seed(seed)
    z = (2.5 * torch.randn((n + 1, vocab), generator=gen, device=DEV)).to(torch.bfloat16)
    y = torch.randint(0, vocab, (n + 1,), generator=gen, device=DEV)
    logp = torch.log_softmax(z.double() * scale, 1).gather(1, y[:, None])[:, 0]
    sums = torch.stack([logp[:n].sum(), logp[n]])
    ref = sums.float()
    got = dx.detox_preference_loss(z, y, torch.tensor([0, n, n + 1], dtype=torch.int32, device=DEV), ref, beta=beta, scale=scale, want_grad=False)
    gap = sums - ref.double()
    want = beta * float(gap[0] - gap[1])
    assert abs(float(got.margin[0]) - want) <= beta * (n + 1) * (1e-8 + 3.6e-8) + 2 * U * abs(want)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("scale", SCALES)
@pytest.mark.parametrize("vocab", [200, 3001, 40000])
def test_the_ratio_of_a_token_that_is_far_off(dtype, scale, vocab):
    """Log-probabilities of thousands, whose difference to the old ones is what counts.  The sum of the others is off by a few units (their exponents, within 15 of the
    largest, twice 2^-24 of that; powers 2^-22; fewer than 100 additions; 1e-7 for the temperature of their distances); then about 20 roundings."""
    n = 9
    gen = torch.Generator(device=DEV).manual_seed(vocab)
    z = torch.randn((n, vocab), generator=gen, device=DEV)
    z[3:] += 1000.0                                # common offsets do not matter
    z = z.to(dtype)
    y = torch.randint(0, vocab, (n,), generator=gen, device=DEV)
    z[torch.arange(n, device=DEV), y] = -torch.tensor([30.0, 300.0, 2000.0, 3.0, 7.0, 50.0, 700.0, 5000.0, 20000.0], device=DEV).to(dtype)
    scale32 = float(torch.tensor(scale))
    x = z.double() * scale32
    p = torch.log_softmax(x, 1)
    logp = p.gather(1, y[:, None])[:, 0]
    old = (logp + 0.05).float()
    a, w = torch.ones(n, device=DEV), torch.full((n,), 0.125, device=DEV)
    one = dx.detox_policy_loss(z, y, old, a, None, w, scale=scale32)
    ratio = torch.exp(logp - old.double())
    held = ratio.clamp(0.8, 1.2)
    unit = U * (200 + 4 * 1.5 * 15) + 1e-7
    assert abs(float(one.loss) + 0.125 * float(torch.minimum(ratio, held).sum())) <= 0.125 * n * 1.2 * unit
    inside = (ratio > 0.8) & (ratio < 1.19)
    want = -0.125 * ratio * scale32                # of the chosen entry, whose p is nothing
    got = one.dz.gather(1, y[:, None])[:, 0].double()
    assert bool(((got - want).abs() <= want.abs() * (unit + torch.finfo(dtype).eps / 2 * 1.01))[inside].all())
    # and the KL term's, with the reference as near
    ref = (logp - 0.3).float()
    two = dx.detox_policy_loss(z, y, old, 0 * a, ref, w, kl_coef=1.0, scale=scale32)
    d = ref.double() - logp
    kl = torch.expm1(d) - d
    assert abs(float(two.kl) - 0.125 * float(kl.sum())) <= 0.125 * n * (2 * unit + 4 * U)
    want = 0.125 * -torch.expm1(d) * scale32
    got = two.dz.gather(1, y[:, None])[:, 0].double()
    assert bool(((got - want).abs() <= 0.125 * scale32 * 2 * unit + want.abs() * torch.finfo(dtype).eps / 2 * 1.01).all())
