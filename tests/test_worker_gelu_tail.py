"""gelu and its derivative far to the left, where the distribution function is small: relative to their own size."""
import math

import pytest
import torch

import paper_1907_12205_b200 as dx

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
F16, BF16, F32 = torch.float16, torch.bfloat16, torch.float32
HALF_UNIT = {F16: 2.0 ** -11, BF16: 2.0 ** -8}
TINY = {F16: 2.0 ** -25, BF16: 2.0 ** -134}      # half the smallest step
# The factor that decides is exp(-g^2 / 2): an argument of 32 that is off by 2^-23 of itself moves it by 3.8e-6, and so does erfc's
# argument, off by as much, by 7.6e-6.  2^-15 covers either way to compute it.
SLACK = 2.0 ** -15


def reference(g):
    c = 0.5 * torch.erfc(-g / math.sqrt(2))
    return g * c, c + g * torch.exp(-g * g / 2) / math.sqrt(2 * math.pi)


def near(got, ref, dtype, what):
    got, ref = got.cpu().double(), ref.double()
    bound = (HALF_UNIT[dtype] * (1 + SLACK) + SLACK) * ref.abs() + TINY[dtype]
    bad = (got - ref).abs() > bound
    assert not bad.any(), f"{what}: {int(bad.sum())} of {bad.numel()} off, worst {float(((got - ref).abs() / bound).max())} bounds"


@pytest.mark.parametrize("tokens", [1, 2100])
@pytest.mark.parametrize("dtype", [F16, BF16])
def test_the_negative_tail(dtype, tokens):
    """One token, g = a row of weights from -3 to -8, u = 1 (and the same for many tokens, in pairs of CTAs)."""
    g = torch.arange(-8 * 32, -3 * 32 + 1, dtype=torch.float64) / 32     # exact in both types
    hidden = g.numel()
    x = torch.ones((tokens, 2), dtype=torch.float64)
    wg, wu = torch.zeros((hidden, 2), dtype=torch.float64), torch.zeros((hidden, 2), dtype=torch.float64)
    wg[:, 0], wu[:, 1] = g, 1.0
    x, wg, wu = (t.to(dtype).to(DEV) for t in (x, wg, wu))
    a, da = reference(g)
    h, kept = dx.detox_gated(x, wg, wu, dx.ACT_GELU, keep=True)
    near(h, a.expand(tokens, hidden), dtype, "h")
    # the gradients of one token alone: dWu = act(g), dWg = act'(g), rounded to the type
    one = dx.Kept(kept.q[:, :1], kept.e[:, :1])
    taken = (kept.gq[:1].float() * kept.ge[:1].float().repeat_interleave(128, 1)[:, :hidden]).cpu().double()[0]
    dh = torch.ones((1, hidden), dtype=dtype, device=DEV)
    for k, at in ((None, g), (one, taken)):
        a, da = reference(at)
        _, dwg, dwu = dx.detox_gated_backward(dh, x[:1], wg, wu, dx.ACT_GELU, kept=k, dw_dtype=F32)
        near(dwu[:, 1], a, dtype, "dwu")
        near(dwg[:, 0], da, dtype, "dwg")
