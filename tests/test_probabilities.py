"""The probabilities in the gradients behind a forward pass: as near as the log-sum-exp that is handed over allows, whatever its size."""
import pytest
import torch

import paper_1907_12205_b200 as dx

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TYPES = [torch.bfloat16, torch.float16, torch.float32]
U = 2.0 ** -24
TINY = {torch.bfloat16: 2.0 ** -126, torch.float16: 2.0 ** -25, torch.float32: 2.0 ** -126}


def inputs(rows, vocab, dtype, offset, size):
    gen = torch.Generator(device=DEV).manual_seed(vocab)
    z = (size * torch.randn((rows, vocab), generator=gen, device=DEV) + offset).to(dtype)
    return z, torch.randint(0, vocab, (rows,), generator=gen, device=DEV)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("scale", [1.0, 0.7, 1.3])
@pytest.mark.parametrize("offset", [0.0, 700.0, -3000.0, 20000.0])
def test_the_gradient_is_the_formulas_for_the_lse_that_it_is_given(dtype, scale, offset):
    """exp(scale z - lse) of the fp32 lse: an exponent rounded once, to 2^-24 of its own size, and short of the temperature's second part times that; a power
    (2^-22), its factor and two products."""
    z, y = inputs(17, 1203, dtype, offset, 2.0)
    scale = float(torch.tensor(scale))
    lse = dx.detox_token_logp(z, y, scale=scale).lse
    d = torch.randn(17, device=DEV, generator=torch.Generator(device=DEV).manual_seed(1))
    got = dx.detox_token_logp_backward(d, z, y, lse, scale=scale).double()
    x = z.double() * scale - lse.double()[:, None]
    p = torch.exp(x)
    own = torch.zeros_like(p).scatter_(1, y[:, None], 1.0)
    want = scale * d.double()[:, None] * (own - p)
    unit = U * (12 + 3 * x.abs())
    bound = scale * d.double().abs()[:, None] * (p * unit + 2 * U * own) + want.abs() * torch.finfo(dtype).eps / 2 * 1.01 + TINY[dtype]
    assert bool(((got - want).abs() <= bound).all())


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("scale", [1.0, 1.3])
@pytest.mark.parametrize("offset", [0.0, 700.0, 20000.0])
@pytest.mark.parametrize("vocab", [300, 2049, 33000])
def test_the_preference_gradient_does_not_depend_on_a_common_offset(dtype, scale, offset, vocab):
    """Its probabilities come from a log-sum-exp of more than fp32's bits: off by the sum (fewer than 100 additions, powers) and an exponent's rounding."""
    rows, beta = 12, 0.2
    z, y = inputs(rows, vocab, dtype, offset, 2.0)
    scale = float(torch.tensor(scale))
    x = z.double() * scale
    logp = torch.log_softmax(x, 1)
    own = torch.zeros_like(logp).scatter_(1, y[:, None], 1.0)
    mine = logp.gather(1, y[:, None])[:, 0]
    ref = torch.stack([mine[:7].sum(), mine[7:].sum()]).float()
    got = dx.detox_preference_loss(z, y, torch.tensor([0, 7, 12], dtype=torch.int32, device=DEV), ref, beta=beta, scale=scale, grad_scale=3.0)
    h = beta * ((mine[:7].sum() - ref[0].double()) - (mine[7:].sum() - ref[1].double()))
    dh = -3.0 * beta * torch.sigmoid(-h)
    coef = torch.where(torch.arange(rows, device=DEV) < 7, dh, -dh)[:, None] * scale
    want = coef * (own - torch.exp(logp))
    unit = U * (140 + 6 * (x - x.amax(1, keepdim=True)).abs())
    bound = coef.abs() * torch.exp(logp) * unit + want.abs() * (40 * U + torch.finfo(dtype).eps / 2 * 1.01) + TINY[dtype]
    assert bool(((got.dz.double() - want).abs() <= bound).all())


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("vocab", [60, 3000])
def test_the_preference_gradient_of_a_sure_token(dtype, vocab):
    """1 - p of the chosen token to a few units of itself, however small."""
    rows = 24
    z, y = inputs(rows, vocab, dtype, 0.0, 1.0)
    z[torch.arange(rows, device=DEV), y] = torch.linspace(0, 40, rows, device=DEV).to(dtype)
    x = z.double()
    q = torch.exp(x - x.gather(1, y[:, None])).scatter(1, y[:, None], 0.0).sum(1)
    mine, rest = -torch.log1p(q), q / (1 + q)
    ref = torch.stack([mine[:12].sum(), mine[12:].sum()]).float()
    got = dx.detox_preference_loss(z, y, torch.tensor([0, 12, 24], dtype=torch.int32, device=DEV), ref, beta=0.1)
    h = 0.1 * ((mine[:12].sum() - ref[0].double()) - (mine[12:].sum() - ref[1].double()))
    dh = -0.1 * torch.sigmoid(-h)
    want = torch.where(torch.arange(rows, device=DEV) < 12, dh, -dh) * rest
    own = got.dz.gather(1, y[:, None])[:, 0].double()
    assert bool(((own - want).abs() <= want.abs() * (U * (180 + 4 * 50) + torch.finfo(dtype).eps / 2 * 1.01) + TINY[dtype]).all())
