"""The gated products' bounded waits: what a wait that runs out leaves behind."""
import os
import re

import pytest
import torch

import paper_1907_12205_b200 as dx

DEV = "cuda:0"
BF16, F32 = torch.bfloat16, torch.float32


def inputs(tokens, in_dim, hidden, dtype=BF16, seed=0):
    gen = torch.Generator(device=DEV).manual_seed(seed)
    shapes = ((tokens, in_dim), (hidden, in_dim), (hidden, in_dim), (tokens, hidden))
    x, wg, wu, dh = (torch.randn(s, generator=gen, device=DEV) for s in shapes)
    return x.to(dtype), (wg * in_dim ** -0.5).to(dtype), (wu * in_dim ** -0.5).to(dtype), dh.to(dtype)


@pytest.fixture
def short_limit():
    """Ten thousand clocks, some six microseconds.  (A wait looks at the clock only after the hardware has suspended it for a while, so the
    accumulators of the products here take 45 us and more.)"""
    assert dx.gated_expired_waits(clear=True)[0] == 0
    yield lambda: dx.gated_wait_limit(10_000)
    torch.cuda.synchronize()
    dx.gated_wait_limit(0)
    dx.gated_expired_waits(clear=True)


# what the shape rule takes for them: CTAs that multiply a tile, its columns, CTAs that share its reduction
FORWARD = [((3, 65536, 300), False, (1, 128, 8)), ((3, 65536, 300), True, (1, 256, 8)), ((1280, 16384, 1800), False, (1, 128, 1)),
           ((1152, 16384, 1024), True, (1, 256, 2)), ((2048, 16384, 4096), False, (2, 256, 1)), ((2048, 16384, 4096), True, (2, 256, 1))]


@pytest.mark.gpu
@pytest.mark.parametrize("sizes,keep,shape", FORWARD)
def test_a_forward_wait_that_runs_out_is_reported_and_the_next_call_is_right(short_limit, sizes, keep, shape):
    x, wg, wu, _ = inputs(*sizes)
    call = lambda **kw: dx.detox_gated(x, wg, wu, keep=keep, **kw)  # noqa: E731
    want = call()
    ws = torch.empty(dx.detox_gated_workspace_bytes(x, wg, wu), dtype=torch.uint8, device=DEV)
    h = torch.zeros_like(want[0] if keep else want)
    short_limit()
    got = call(h=h, ws=ws)
    assert dx.read_status(ws) == 5
    with pytest.raises(dx.DetoxError):
        dx.check_status(ws)
    count, first = dx.gated_expired_waits()
    assert count > 0 and (first.form, first.ctas, first.columns, first.split) == (0, *shape)
    assert 0 <= first.rank < max(first.ctas, first.split) and 0 <= first.barrier < 4
    assert bool(h.isnan().all())                       # no output that could be taken for a result
    if keep:
        assert bool(got[1].q.float().isnan().all()) and bool((got[1].e.view(torch.uint8) == 127).all())
    dx.gated_wait_limit(0)
    again = call(h=h, ws=ws)
    assert dx.read_status(ws) == 0
    assert torch.equal(h, want[0] if keep else want)
    if keep:
        for a, b in zip(again[1], want[1]):
            assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))
    assert dx.gated_expired_waits(clear=True)[0] == count and dx.gated_expired_waits() == (0, None)


@pytest.mark.gpu
@pytest.mark.parametrize("sizes", [(2048, 16384, 8192), (1000, 16384, 9600), (64, 32768, 9000)])
@pytest.mark.parametrize("kept", [False, True])
def test_a_backward_wait_that_runs_out_ends_the_call(short_limit, sizes, kept):
    x, wg, wu, dh = inputs(*sizes)
    k = dx.detox_gated(x, wg, wu, keep=True)[1] if kept else None
    want = dx.detox_gated_backward(dh, x, wg, wu, kept=k, dw_dtype=F32)
    outs = [torch.zeros_like(t) for t in want]
    ws = torch.empty(dx.detox_gated_backward_workspace_bytes(x, wg, wu, kept=k), dtype=torch.uint8, device=DEV)
    short_limit()
    dx.detox_gated_backward(dh, x, wg, wu, kept=k, dx=outs[0], dwg=outs[1], dwu=outs[2], ws=ws)
    assert dx.read_status(ws) == 5
    assert dx.gated_expired_waits()[1].form == (2 if kept else 1)
    # the later products read what the first one left undone: they give up, whatever their own waits would have done
    assert all(bool(t.isnan().all()) for t in outs[(1 if kept else 0):]) and bool(outs[0].isnan().any())
    dx.gated_wait_limit(0)
    dx.detox_gated_backward(dh, x, wg, wu, kept=k, dx=outs[0], dwg=outs[1], dwu=outs[2], ws=ws)
    assert dx.read_status(ws) == 0
    assert all(torch.equal(a, b) for a, b in zip(outs, want))


@pytest.mark.gpu
def test_an_expired_wait_is_known_without_a_workspace(short_limit):
    """Calls that make their own workspace take its status word with them; the count stays, over later calls too."""
    x, wg, wu, _ = inputs(2048, 16384, 4096)
    short_limit()
    dx.detox_gated(x, wg, wu)
    dx.gated_wait_limit(0)
    dx.detox_gated(x, wg, wu)
    assert dx.gated_expired_waits()[0] > 0


def test_the_limit_and_the_count_need_no_workspace():
    from paper_1907_12205_b200 import build
    build.build()
    assert dx.gated_wait_limit() == 0 and dx.gated_wait_limit(5000) == 0 and dx.gated_wait_limit(20_000) == 0
    assert dx.gated_wait_limit(9_999) == 20_000 and dx.gated_wait_limit(0) == 20_000 and dx.gated_wait_limit() == 0
    header = open(os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include", "detox.h")).read()
    words = {k: int(v) for k, v in re.findall(r"#define (DETOX_EXPIRED_WORDS|DETOX_WAIT_LIMIT_MIN) (\d+)", header)}
    assert words == {"DETOX_EXPIRED_WORDS": len(dx.ExpiredWait._fields), "DETOX_WAIT_LIMIT_MIN": 10_000}
