"""Long series of steps of the gated products: every one finishes, with the same bits."""
import pytest
import torch

import paper_1907_12205_b200 as dx

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
F16, BF16 = torch.float16, torch.bfloat16

# forward, dx and weight gradients all in pairs of CTAs; forward and weight gradients; forward; forward and one split
SERIES = [(8192, 2048, 5632, BF16, dx.ACT_SILU, True, 400), (1001, 1000, 2730, F16, dx.ACT_SILU, False, 1000),
          (2300, 640, 1920, BF16, dx.ACT_GELU, True, 1000), (500, 512, 1408, BF16, dx.ACT_GELU, True, 2000)]


@pytest.mark.parametrize("tokens,in_dim,hidden,dtype,act,kept,steps", SERIES)
def test_steps_one_after_another_all_finish_with_the_same_bits(tokens, in_dim, hidden, dtype, act, kept, steps):
    """A full batch's products run as pairs of CTAs, one behind the other; they stopped making progress about once in some thousand
    steps while they took part in the chain of overlapping launches."""
    gen = torch.Generator(device=DEV).manual_seed(0)
    shapes = ((tokens, in_dim), (hidden, in_dim), (hidden, in_dim), (tokens, hidden))
    x, wg, wu, dh = (torch.randn(s, generator=gen, device=DEV) for s in shapes)
    x, wg, wu, dh = x.to(dtype), (wg * in_dim ** -0.5).to(dtype), (wu * in_dim ** -0.5).to(dtype), dh.to(dtype)
    forward_ws = torch.empty(dx.detox_gated_workspace_bytes(x, wg, wu), dtype=torch.uint8, device=DEV)
    pair = dx.detox_checkpoint_pack(x) if kept else x
    ws = torch.empty(dx.detox_gated_backward_workspace_bytes(pair, wg, wu, act), dtype=torch.uint8, device=DEV)

    def step():
        k, xin = None, x
        if kept:
            k = dx.detox_gated(x, wg, wu, act, keep=True, ws=forward_ws)[1]
            xin = dx.detox_checkpoint_pack(x)
        return dx.detox_gated_backward(dh, xin, wg, wu, act, kept=k, ws=ws)

    first = [t.clone() for t in step()]
    for i in range(steps):
        got = step()
        if i % 50 == 49:
            if kept:
                dx.check_status(forward_ws, f"after {i + 1} steps")
            dx.check_status(ws, f"after {i + 1} steps")
            assert all(torch.equal(a, b) for a, b in zip(first, got)), f"after {i + 1} steps"
