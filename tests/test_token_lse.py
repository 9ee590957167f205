"""The log-sum-exp of every row, whether a token was chosen there or not, against 64 bits."""
import pytest
import torch

import paper_1907_12205_b200 as dx

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TYPES = [torch.bfloat16, torch.float16, torch.float32]
U = 2.0 ** -24
INF, NAN = float("inf"), float("nan")


def logits(rows, vocab, dtype, pad=0, offset=0, size=3.0):
    gen = torch.Generator(device=DEV).manual_seed(rows + vocab)
    flat = (size * torch.randn(rows * (vocab + pad) + offset, generator=gen, device=DEV)).to(dtype)
    return flat[offset:].view(rows, vocab + pad)[:, :vocab], torch.randint(0, vocab, (rows,), generator=gen, device=DEV)


def slack(z, scale):
    """Exponents: a factor and a product rounded, twice 2^-24 of the row's range and of its largest entry's size; powers and logarithm: 2^-22 and a few units; sums: fewer
    than 100 additions one after another."""
    x = z.double() * scale
    return U * (120 + 6 * (x.amax(1) - x.amin(1)) + 6 * x.abs().amax(1))


def check(rows, vocab, dtype, chosen, pad, offset, scale, index):
    z, y = logits(rows, vocab, dtype, pad, offset)
    gone = ~torch.tensor([chosen(i) for i in range(rows)], device=DEV)
    y = torch.where(gone, torch.tensor([-1, -100], device=DEV)[torch.arange(rows, device=DEV) % 2], y).to(index)
    x = z.double() * scale
    lse = torch.logsumexp(x, 1)
    logp = torch.where(gone, 0.0, x.gather(1, y.clamp(min=0).long()[:, None])[:, 0] - lse)
    got = dx.detox_token_logp(z, y, scale=scale)
    assert bool(((got.lse.double() - lse).abs() <= slack(z, scale)).all())
    assert bool(((got.logp.double() - logp).abs() <= slack(z, scale)).all()) and bool((got.logp[gone] == 0).all())
    alone = dx.detox_token_logp(z, y, scale=scale, want_lse=False)
    assert alone.lse is None and torch.equal(alone.logp, got.logp)
    # and a gradient's rows stay zero where no token was chosen
    dz = dx.detox_token_logp_backward(torch.ones(rows, device=DEV), z, y, got.lse, scale=scale)
    assert bool((dz[gone] == 0).all()) and (vocab == 1 or bool((dz[~gone] != 0).any(1).all()))


ROWS = [lambda i: False, lambda i: i % 2 == 0, lambda i: i % 10 != 3]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,vocab", [(1, 1), (5, 7), (40, 256), (33, 1000), (9, 2051), (160, 5000), (3, 8000), (301, 10007)])
@pytest.mark.parametrize("which", range(len(ROWS)))
def test_every_row_has_its_log_sum_exp(dtype, rows, vocab, which):
    for pad, offset, scale, index in ((0, 0, 1.0, torch.int64), (5, 3, 1.25, torch.int32)):
        check(rows, vocab, dtype, ROWS[which], pad, offset, scale, index)


@pytest.mark.parametrize("dtype", TYPES)
def test_rows_that_are_masked_infinite_or_nan(dtype):
    z, _ = logits(6, 300, dtype)
    z[0] = -INF
    z[1, 1:] = -INF
    z[2, 7] = NAN
    z[3] = INF
    y = torch.tensor([-1, -1, -1, -1, 5, -1], device=DEV)
    got = dx.detox_token_logp(z, y)
    want = torch.logsumexp(z.double(), 1)
    assert float(got.lse[0]) == -INF and bool(got.lse[2:4].isnan().all())
    assert bool(((got.lse.double() - want)[[1, 4, 5]].abs() <= 200 * U).all())
    assert bool((got.logp[[0, 1, 2, 3, 5]] == 0).all()) and bool(got.logp.isfinite().all())
    # not read where only the log-probabilities are wanted, and not looked at by the gradient
    assert torch.equal(dx.detox_token_logp(z, y, want_lse=False).logp, got.logp)
    dz = dx.detox_token_logp_backward(torch.ones(6, device=DEV), z, y, got.lse)
    assert bool((dz[[0, 1, 2, 3, 5]] == 0).all()) and bool(dz[4].isfinite().all())


def gradient_bound(exact, d, p, y, scale, dtype, off):
    """A rounding to the type; two roundings of the coefficient; the probabilities' relative error."""
    own = torch.zeros_like(p).scatter_(1, y.clamp(min=0)[:, None].long(), 1.0)
    near = (own - p).abs() * 2 * U * d.abs()[:, None] + d.abs()[:, None] * (p * off[:, None] + 4 * U * (own + p))
    tiny = {torch.bfloat16: 2.0 ** -134, torch.float16: 2.0 ** -25, torch.float32: 2.0 ** -126}[dtype]
    return exact.abs() * torch.finfo(dtype).eps / 2 * 1.001 + 1.01 * scale * near + tiny


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,vocab", [(3, 2), (5, 7), (9, 100), (40, 256), (33, 1000), (70, 2051), (4, 4099), (300, 3001), (3, 8200), (5, 16390), (7, 32770),
                                        (160, 5000), (80, 50257), (3, 131072), (4, 262144)])
def test_the_gradient_of_a_batch_with_rows_without_a_token(dtype, rows, vocab):
    for pad, offset, scale, index in ((0, 0, 1.0, torch.int64), (5, 3, 0.7, torch.int32)):
        z, y = logits(rows, vocab, dtype, pad, offset)
        y[1], y[0] = -1, vocab - 1
        y = y.to(index)
        x = z.double() * scale
        lse = torch.logsumexp(x, 1)
        got = dx.detox_token_logp(z, y, scale=scale)
        off = slack(z, scale)
        assert bool(((got.lse.double() - lse).abs() <= off).all())
        d = torch.randn(rows, device=DEV, generator=torch.Generator(device=DEV).manual_seed(3))
        if rows > 4:
            d[2] = 0.0
        dz = dx.detox_token_logp_backward(d, z, y, got.lse, scale=scale)
        p = torch.exp(x - lse[:, None])
        exact = -p * d.double()[:, None]
        exact.scatter_add_(1, y.clamp(min=0)[:, None].long(), d.double()[:, None])
        exact = torch.where((y >= 0)[:, None], exact, 0.0) * scale
        # the rounding of lse to fp32 enters every probability
        assert bool(((dz.double() - exact).abs() <= gradient_bound(exact, d.double(), p, y, scale, dtype, 2 * off + 2 * U * lse.abs())).all())
        assert bool((dz[1] == 0).all()) and (rows <= 4 or bool((dz[2] == 0).all()))
        z2 = torch.empty_strided(z.shape, z.stride(), dtype=dtype, device=DEV).copy_(z)   # in place
        assert torch.equal(dx.detox_token_logp_backward(d, z2, y, got.lse, scale=scale, dz=z2), dz) and torch.equal(z2, dz)
