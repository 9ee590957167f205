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


@pytest.mark.parametrize("bits", BITS)
def test_the_least_eps_beside_gradients_that_are_zero_or_next_to_it(bits):
    """Entries without a gradient stay as they are, and a direction is m / (root + eps) however small.  The direction is off by 2^-20, and by what v, its square and the
    product are rounded to where fp32 has steps of 2^-149 alone: three of those.  (8 bits: v below 2^-126 is 0, and the least eps larger.)"""
    n, eps, b1, b2 = 4096, 1e-18 if bits == 32 else 1e-15, 0.9, 0.999
    gen = torch.Generator(device=DEV).manual_seed(1)
    g = torch.randn(n, generator=gen, device=DEV) * torch.pow(10.0, -22 + 6 * torch.rand(n, generator=gen, device=DEV))
    g[::3] = 0.0
    start = torch.randn(n, generator=gen, device=DEV) * 1e-3
    for gradient in (g, torch.zeros_like(g)):
        p = start.clone()
        m, v = dx.detox_adamw_state([p], bits)
        dx.detox_adamw([p], [gradient], m, v, 1, 1.0, beta1=b1, beta2=b2, eps=eps)
        g64 = gradient.double()
        square = (1 - b2) * g64 * g64
        root, c2 = torch.sqrt(square), (1 - b2) ** 0.5
        way = g64 / (root / c2 + eps)
        off = (torch.sqrt(square + 3 * 2.0 ** -149) - torch.sqrt((square - 3 * 2.0 ** -149).clamp(min=0.0))) / c2
        if bits == 8:
            off = torch.where(square < 1.01 * 2.0 ** -126, 1.01 * 2.0 ** -63 / c2, off)
        low = (root / c2 + eps - off).clamp(min=eps)
        bound = way.abs() * (2.0 ** -20 + off / low) + 2.0 ** -23 * (way.abs() + start.abs())
        assert bool(((start.double() - p.double() - way).abs() <= bound).all())
        assert torch.equal(p[::3], start[::3])


def test_an_eps_that_is_too_small_is_refused():
    p = torch.zeros(64, device=DEV)
    m, v = dx.detox_adamw_state([p])
    for eps in (9e-19, 1e-38, 1e-46, 5e-324, 0.0, float("nan")):
        with pytest.raises(dx.DetoxError):
            dx.detox_adamw([p], [p + 1], m, v, 1, 0.1, eps=eps)
    m8, v8 = dx.detox_adamw_state([p], 8)
    with pytest.raises(dx.DetoxError):
        dx.detox_adamw([p], [p + 1], m8, v8, 1, 0.1, eps=9e-16)
    dx.detox_adamw([p], [p + 1], m8, v8, 1, 0.0, eps=1e-15)
    dx.detox_adamw([p], [p + 1], m, v, 1, 0.1, eps=1e-18)
    assert bool(((p + 0.1).abs() <= 1e-6).all())


def test_what_is_stepped_twice_or_read_as_a_gradient_is_refused():
    new = lambda: torch.zeros(300, device=DEV)  # noqa: E731
    p, q, g = new(), new(), new() + 1
    m, v = dx.detox_adamw_state([p, q], 8)
    dx.detox_adamw([p, q], [g, g], m, v, 1, 0.1)                         # one gradient for both is fine
    for bad_m, bad_v in (([m[0], (m[1][0], m[0][1])], v), (m, [v[0], (v[1][0], v[0][1])]), (m, [(v[0][0], m[0][1]), v[1]])):
        with pytest.raises(ValueError, match="twice"):
            dx.detox_adamw([p, q], [g, g], bad_m, bad_v, 1, 0.1)
    m, v = dx.detox_adamw_state([p, q])
    for grads in ([g, p], [q, g], [g, m[0]], [v[1], g]):
        with pytest.raises(ValueError, match="stepped"):
            dx.detox_adamw([p, q], grads, m, v, 1, 0.1)
    empty = torch.empty(0, device=DEV)
    dx.detox_adamw([p, empty], [g, empty], [m[0], empty], [v[0], empty], 1, 0.1)
