"""The optimizer's step at the edges of its arguments."""
import pytest
import torch

import paper_1907_12205_b200 as dx

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BITS = [32, 8]


def flat(state):
    return [t for x in state for t in (x if isinstance(x, tuple) else (x,))]


def same(a, b):
    return all(torch.equal(x.view(torch.uint8), y.view(torch.uint8)) for x, y in zip(a, b))


@pytest.mark.parametrize("bits", BITS)
def test_a_step_from_the_device_that_is_below_1_is_the_first(bits):
    """Weights and states, whose random bits depend on the step's number."""
    gen = torch.Generator(device=DEV).manual_seed(0)
    start, g = torch.randn(9000, generator=gen, device=DEV), torch.randn(9000, generator=gen, device=DEV)
    results = []
    for step in (1, 0, -1, -2 ** 40):
        p = start.clone()
        m, v = dx.detox_adamw_state([p], bits)
        for x in flat(m) + flat(v):
            if x.dtype == torch.float8_e4m3fn:
                x.view(torch.uint8).fill_(0x30)        # 0.5: there is something to round
        dx.detox_adamw([p], [g], m, v, torch.full((1,), step, dtype=torch.int64, device=DEV), 0.1, seed=5)
        results.append([p] + flat(m) + flat(v))
    assert all(same(r, results[0]) for r in results[1:])
    p = start.clone()
    m, v = dx.detox_adamw_state([p], bits)
    dx.detox_adamw([p], [g], m, v, torch.full((1,), 2, dtype=torch.int64, device=DEV), 0.1, seed=5)
    assert not torch.equal(p, results[0][0])
