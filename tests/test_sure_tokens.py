"""Tokens that a row is sure of: log-probabilities near 0 and gradients near 0 keep their bits, which a sum that has the chosen token's own power in it would swallow."""
import pytest
import torch

import paper_1907_12205_b200 as dx

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TYPES = [torch.bfloat16, torch.float16, torch.float32]
U = 2.0 ** -24
TINY = {torch.bfloat16: 2.0 ** -126, torch.float16: 2.0 ** -25, torch.float32: 2.0 ** -126}


def sure_rows(rows, vocab, dtype, pad, offset):
    """Rows whose chosen token leads by 0 to 60."""
    gen = torch.Generator(device=DEV).manual_seed(vocab)
    flat = torch.randn(rows * (vocab + pad) + offset, generator=gen, device=DEV).to(dtype)
    z = flat[offset:].view(rows, vocab + pad)[:, :vocab]
    y = torch.randint(0, vocab, (rows,), generator=gen, device=DEV)
    z[torch.arange(rows, device=DEV), y] = torch.linspace(0, 60, rows, device=DEV).to(dtype)
    return z, y


def exact(z, y, scale):
    """log p and 1 - p of the chosen tokens, from the others' sum alone."""
    x = z.double() * scale
    own = x.gather(1, y[:, None])
    q = torch.exp(x - own).scatter(1, y[:, None], 0.0).sum(1)
    return -torch.log1p(q), q / (1 + q)


def relative(z, scale):
    """q's error relative to itself: of an exponent two roundings of up to its size (the distance of the largest entries, 70 here, in which the chosen one lies) and of the numbers
    that it is the difference of; powers 2^-22 and two more factors; fewer than 100 additions."""
    x = z.double() * scale
    return U * (140 + 4 * (x.amax(1) - x.amin(1)) + 4 * x.abs().amax(1))


SHAPES = [(40, 2), (61, 30), (40, 129), (33, 2000), (61, 2051), (300, 5003), (21, 8200), (9, 33000), (3, 131072), (160, 32000)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,vocab", SHAPES)
def test_log_probabilities_near_zero(dtype, rows, vocab):
    for pad, offset, scale in ((0, 0, 1.0), (3, 1, 0.8)):
        z, y = sure_rows(rows, vocab, dtype, pad, offset)
        logp, rest = exact(z, y, scale)
        off = relative(z, scale)
        got = dx.detox_token_logp(z, y, scale=scale).logp
        w = torch.full((rows,), 0.5, device=DEV)
        old = (logp + 0.01).float()
        pol = dx.detox_policy_loss(z, y, old, -w, None, w, scale=scale, grad_scale=2.0)
        for one in (got, pol.logp):
            assert bool(((one.double() - logp).abs() <= logp.abs() * (off + U)).all())
            assert bool((one[logp < -2.0 ** -120] < 0).all())
        # the gradient of the chosen entry is its coefficient times 1 - p: q's error in 1 - p and in the ratio p / e^old, and roundings
        coef = 0.5 * torch.exp(logp - old.double()) * scale
        want = coef * rest
        own = pol.dz.gather(1, y[:, None])[:, 0].double()
        assert bool(((own - want).abs() <= want * (2 * off + 40 * U + torch.finfo(dtype).eps / 2 * 1.01) + TINY[dtype]).all())
        # and that of the others p_j times it
        p = torch.softmax(z.double() * scale, 1).scatter(1, y[:, None], 0.0)
        others = pol.dz.double().scatter(1, y[:, None], 0.0)
        want = -coef[:, None] * p
        assert bool(((others - want).abs() <= want.abs() * (3 * off + 40 * U + torch.finfo(dtype).eps / 2 * 1.01)[:, None] + TINY[dtype]).all())


def test_a_row_of_one_entry_and_rows_with_nothing_beside_the_chosen_one():
    for vocab in (1, 9, 3000):
        z = torch.full((4, vocab), float("-inf"), device=DEV)
        y = torch.tensor([0, vocab - 1, vocab // 2, 0], device=DEV)
        z[torch.arange(4, device=DEV), y] = torch.tensor([0.0, -3.5, 1e4, 7.0], device=DEV)
        one = torch.ones(4, device=DEV)
        got = dx.detox_token_logp(z, y)
        pol = dx.detox_policy_loss(z, y, 0 * one, one, None, one)
        assert bool((got.logp == 0).all()) and bool((pol.logp == 0).all()) and bool((pol.dz == 0).all())
        assert bool(((got.lse - torch.tensor([0.0, -3.5, 1e4, 7.0], device=DEV)).abs() <= 1e4 * U).all()) and float(pol.loss) == -4.0
