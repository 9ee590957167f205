"""The range of the gradients of g and u, which are rounded to the operands' type between the two backward products."""
import pytest
import torch

import paper_1907_12205_b200 as dx

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
F16, BF16, F32 = torch.float16, torch.bfloat16, torch.float32


def problem(tokens, dtype, scale):
    """Whole numbers, relu: du = dh g and dg = dh u for g > 0.  Every entry of dh is 0 or `scale`, a power of two."""
    gen = torch.Generator().manual_seed(tokens)
    in_dim, hidden = 16, 200
    x = torch.randint(1, 3, (tokens, in_dim), generator=gen).double()
    wg, wu = (torch.randint(0, 2, (hidden, in_dim), generator=gen).double() for _ in range(2))
    wg[:, 0] = wu[:, 1] = 1.0
    dh = torch.randint(0, 2, (tokens, hidden), generator=gen).double()
    g, u = x @ wg.T, x @ wu.T
    dg, du = dh * u, dh * g
    ref = (dg @ wg + du @ wu, dg.T @ x, du.T @ x)
    return [t.to(dtype).to(DEV) for t in (dh * scale, x, wg, wu)], ref, (dg, du)


@pytest.mark.parametrize("kept", [False, True])
@pytest.mark.parametrize("tokens", [3, 300])
def test_a_power_of_two_on_dh_comes_out_again_within_the_range(tokens, kept):
    """Sums of whole numbers below 2^24, times the scale: exact at every scale that keeps dg and du (at most 32) in range."""
    for dtype, scales in ((F16, (-14, 0, 10)), (BF16, (-60, 0, 60))):
        for k in scales:
            (dh, x, wg, wu), ref, _ = problem(tokens, dtype, 2.0 ** k)
            keep = dx.detox_gated(x, wg, wu, dx.ACT_RELU, keep=True)[1] if kept else None
            got = dx.detox_gated_backward(dh, x, wg, wu, dx.ACT_RELU, kept=keep, dw_dtype=F32)
            if kept:                             # g and u as the 8-bit form holds them (whole numbers still)
                g, u = ((q.float() * e.float().repeat_interleave(128, 1)[:, :200]).cpu().double() for q, e in ((keep.gq, keep.ge), (keep.uq, keep.ue)))
                one = dh.cpu().double() / 2.0 ** k
                ref = ((one * u) @ wg.cpu().double() + (one * g) @ wu.cpu().double(), (one * u).T @ x.cpu().double(), (one * g).T @ x.cpu().double())
            assert torch.equal(got[1].cpu().double(), ref[1] * 2.0 ** k) and torch.equal(got[2].cpu().double(), ref[2] * 2.0 ** k)
            assert torch.equal(got[0].cpu(), (ref[0] * 2.0 ** k).to(dtype))


@pytest.mark.parametrize("tokens", [3, 300])
def test_in_half_what_is_too_large_is_seen_and_what_is_too_small_is_zero(tokens):
    (dh, x, wg, wu), _, (dg, du) = problem(tokens, F16, 2.0 ** 13)       # dg, du >= 8 overflow, and only they
    gx, a, b = dx.detox_gated_backward(dh, x, wg, wu, dx.ACT_RELU, dw_dtype=F32)
    over_g, over_u = dg * 2.0 ** 13 > 65504, du * 2.0 ** 13 > 65504
    assert bool(over_g.any()) and bool(over_u.any())
    assert torch.equal((~a.isfinite()).all(1).cpu(), over_g.any(0)) and torch.equal((~b.isfinite()).all(1).cpu(), over_u.any(0))
    assert torch.equal(a.isfinite().all(1).cpu(), ~over_g.any(0)) and torch.equal(b.isfinite().all(1).cpu(), ~over_u.any(0))
    assert not bool(gx.isfinite()[(over_g | over_u).any(1).to(DEV)].any())
    dh = (dh.double() * 2.0 ** -13).to(F16)                              # ones and zeros again, and then far too small a scale
    tiny = torch.full_like(x, 2.0 ** -13)                                # g, u = 2^-13 times a count up to 16: dg, du of 2^-24 2^-2
    got = dx.detox_gated_backward((dh.double() * 2.0 ** -16).to(F16), tiny, wg, wu, dx.ACT_RELU, dw_dtype=F32)
    assert all(bool((t == 0).all()) for t in got)                        # 16 2^-13 2^-16 = 2^-25, halfway to the smallest step: to even
    x32 = [t.to(BF16) for t in (dh, tiny, wg, wu)]
    got = dx.detox_gated_backward((x32[0].double() * 2.0 ** -16).to(BF16), *x32[1:], dx.ACT_RELU, dw_dtype=F32)
    assert bool((got[1] > 0).any()) and bool((got[2] > 0).any())
