"""The optimizer's step against 64 bits: states in 32 bits and in 8, many tensors, any alignment."""
import math

import pytest
import torch

import paper_1907_12205_b200 as dx

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF16, F16, F32 = torch.bfloat16, torch.float16, torch.float32
HALF = {t: torch.finfo(t).eps / 2 for t in (BF16, F16, F32)}
TINY = {BF16: 2.0 ** -134, F16: 2.0 ** -25, F32: 2.0 ** -126}
U = 2.0 ** -24
B1, B2, EPS = 0.9, 0.999, 1e-8


def vector(n, gen, size=1.0, dtype=F32, offset=0):
    return (size * torch.randn(n + offset, generator=gen, device=DEV)).to(dtype)[offset:]


def mixed(x):
    x = (x ^ (x >> 16)) * 0x85EBCA6B % 2 ** 32
    x = (x ^ (x >> 13)) * 0xC2B2AE35 % 2 ** 32
    return x ^ (x >> 16)


def bits(n, seed, step, key):
    first = mixed(torch.tensor((seed + 0x9E3779B9 * step) % 2 ** 32, device=DEV))
    h = mixed(mixed((first + key) % 2 ** 32) ^ torch.arange(n, device=DEV))
    return (h % 65536).double() / 65536, (h // 65536).double() / 65536


def blocks(x):
    return torch.nn.functional.pad(x, (0, -x.numel() % 128)).view(-1, 128)


def taken(state):
    q, e = state
    return (blocks(q.double()) * e.double()[:, None]).reshape(-1)[: q.numel()]


def exact(p, g, m, v, step, lr, wd):
    m, v = B1 * m + (1 - B1) * g, B2 * v + (1 - B2) * g * g
    step_size = (m / (1 - B1 ** step)) / (torch.sqrt(v / (1 - B2 ** step)) + EPS)
    return p - lr * (wd * p + step_size), m, v, step_size


def check_step(p0, p, master, g, m0, v0, step, lr, wd):
    """p, and the m and v before rounding that it followed; how far p may be off: the direction by 2^-20 (its root and inverse, 2^-22 each, and six roundings),
    relative to the sizes of m's two parts, the rest by a few roundings."""
    want, m, v, way = exact(p0, g, m0, v0, step, lr, wd)
    parts = ((B1 * m0.abs() + (1 - B1) * g.abs()) / (1 - B1 ** step)) / (torch.sqrt(v / (1 - B2 ** step)) + EPS)
    off = lr * parts * 2.0 ** -20 + U * (2 * p0.abs() + want.abs() + 4 * lr * wd * p0.abs())
    if master is not None:
        assert bool(((master.double() - want).abs() <= off).all())
        assert torch.equal(p, master.to(p.dtype))
    else:
        assert bool(((p.double() - want).abs() <= off + HALF[p.dtype] * want.abs() * 1.001 + TINY[p.dtype]).all())
    return m, v


KINDS = [(F32, F32, False), (F32, BF16, False), (BF16, F32, True), (BF16, BF16, True), (BF16, F32, False), (F16, F16, True), (F16, F32, False)]


@pytest.mark.parametrize("ptype,gtype,masters", KINDS)
@pytest.mark.parametrize("offset", [0, 1])
def test_states_in_32_bits(ptype, gtype, masters, offset):
    gen = torch.Generator(device=DEV).manual_seed(1)
    sizes = [1, 5, 127, 128, 129, 1000, 2048, 2049, 4096, 70001, 0]
    wd = [0.1 * (i % 2) for i in range(len(sizes))]
    p = [vector(n, gen, 0.05, ptype, offset) for n in sizes]
    master = [vector(n, gen, 0.05, F32, offset) for n in sizes] if masters else None
    m, v = [vector(n, gen, 1e-3, F32, offset) for n in sizes], [vector(n, gen, 1e-3, F32, offset).square_() for n in sizes]
    for step in (1, 2, 1000):
        g = [vector(n, gen, 2e-3, gtype, offset) for n in sizes]
        before = [[x.double() for x in xs] for xs in (master or p, m, v)]
        dx.detox_adamw(p, g, m, v, step, 1e-2, weight_decay=wd, masters=master, grad_scale=0.5)
        for i in range(len(sizes)):
            g64 = 0.5 * g[i].double()
            want_m, want_v = check_step(before[0][i], p[i], master[i] if masters else None, g64, before[1][i], before[2][i], step, 1e-2, wd[i])
            assert bool(((m[i].double() - want_m).abs() <= 3 * U * (before[1][i].abs() + g64.abs()) + TINY[F32]).all())
            assert bool(((v[i].double() - want_v).abs() <= 4 * U * want_v + TINY[F32]).all())


def check_kept(state, x, r, positive):
    """The kept form of x (known to 2^-20 of itself): the scale, and each entry the neighbour that its random bits say, but for those within that of the border."""
    q, e = state
    n = x.numel()
    top = blocks(x.abs()).amax(1)
    scale = torch.exp2(torch.ceil(torch.log2(torch.clamp(top, min=1e-300) / 448)).clamp(min=-126))
    near = (torch.log2(torch.clamp(top, min=1e-300) / 448) - torch.round(torch.log2(torch.clamp(top, min=1e-300) / 448))).abs() < 2.0 ** -18
    assert bool(((e.double() == scale) | near).all())
    a = x.abs() / e.double().repeat_interleave(128)[:n]
    width = torch.exp2(torch.floor(torch.log2(torch.clamp(a, min=2.0 ** -6))) - 3)
    place = a / width + r
    want = torch.floor(place) * width
    if positive:
        want = torch.where((a > 0) & (want == 0), 2.0 ** -9, want)
    got = q.double().abs()
    border = (place - torch.round(place)).abs() <= 16 * 2.0 ** -20 + 2.0 ** -16   # (a / width is at most 16)
    border |= (torch.log2(torch.clamp(a, min=1e-300)) - torch.round(torch.log2(torch.clamp(a, min=1e-300)))).abs() < 2.0 ** -18
    assert bool(((got == want) | border).all())
    assert bool(((got - want).abs() <= 2 * width + 2.0 ** -9).all())
    assert bool(((q.double() == 0) | (torch.sign(q.double()) == torch.sign(x))).all())


@pytest.mark.parametrize("ptype,gtype,masters", [(F32, F32, False), (BF16, F32, True), (BF16, BF16, False), (F16, F16, True), (F32, F16, False)])
@pytest.mark.parametrize("offset", [0, 1])
def test_states_in_8_bits(ptype, gtype, masters, offset):
    gen = torch.Generator(device=DEV).manual_seed(2)
    sizes = [1, 100, 128, 300, 2048, 5000, 8192, 40003]
    p = [vector(n, gen, 0.05, ptype, offset) for n in sizes]
    master = [vector(n, gen, 0.05, F32, offset) for n in sizes] if masters else None
    state = dx.detox_adamw_state([torch.empty(n + offset, device=DEV) for n in sizes], bits=8)
    m, v = ([(q[offset:], e[: -(-n // 128)]) for (q, e), n in zip(s, sizes)] for s in state)
    for step in (1, 2, 3, 500):
        # entries of very different size, as between a word's row and another's; and zeros
        g = [(vector(n, gen, 1e-3) * torch.exp(3 * vector(n, gen)) * (vector(n, gen) > -1.5)).to(gtype) for n in sizes]
        if offset:
            g = [torch.cat([x[:1], x])[1:] for x in g]
        before = [[x.double() for x in (master or p)], [taken(x) for x in m], [taken(x) ** 2 for x in v]]
        dx.detox_adamw(p, g, m, v, step, 1e-3, weight_decay=0.05, masters=master, seed=12345)
        for i, n in enumerate(sizes):
            want_m, want_v = check_step(before[0][i], p[i], master[i] if masters else None, g[i].double(), before[1][i], before[2][i], step, 1e-3, 0.05)
            rm, rv = bits(n, 12345, step, i)
            check_kept(m[i], want_m, rm, False)
            check_kept(v[i], torch.sqrt(want_v), rv, True)


def test_rounding_at_random_keeps_the_mean():
    """A state that moves by far less than its spacing at each step still gets where the 32-bit one does.  The root's mean over 65536 entries: each of 300 steps adds an
    error of at most a step of the form (1 / 8), unbiased and independent, so the mean is off by less than 6 x sqrt(300) / 8 / 256 of it."""
    n = 65536
    g = torch.full((n,), 1e-3, device=DEV)
    g[::2] *= 1.3
    p8, p32 = torch.zeros(n, device=DEV), torch.zeros(n, device=DEV)
    m8, v8 = dx.detox_adamw_state([p8], bits=8)
    m32, v32 = dx.detox_adamw_state([p32])
    for step in range(1, 301):
        dx.detox_adamw([p8], [g], m8, v8, step, 1e-3, seed=7)
        dx.detox_adamw([p32], [g], m32, v32, step, 1e-3)
    for half in (0, 1):
        root, want = float(taken(v8[0])[half::2].mean()), float(v32[0][half::2].double().sqrt().mean())
        assert abs(root / want - 1) <= 6 * math.sqrt(300) / 8 / 181
        mean, want = float(taken(m8[0])[half::2].mean()), float(m32[0][half::2].double().mean())
        assert abs(mean / want - 1) <= 6 * math.sqrt(10) / 8 / 181      # m forgets in ten steps


def test_a_root_is_never_lost_and_the_step_stays_bounded():
    """Beside an entry 2^30 times as large a root would round to 0, and the next step divide by eps alone."""
    p = torch.zeros(128, device=DEV)
    m, v = dx.detox_adamw_state([p], bits=8)
    g = torch.full((128,), 1e-6, device=DEV)
    g[0] = 1e3
    for step in range(1, 6):
        before = p.clone()
        dx.detox_adamw([p], [g if step == 1 else torch.zeros_like(g)], m, v, step, 1.0, seed=step)
        assert bool((v[0][0].float()[1:] > 0).all())
        assert bool(((p - before).abs() <= 10.0).all())                  # (1 - b1) / sqrt(1 - b2) and the corrections


def test_infinities_and_nan_stay_where_they_are():
    for bits_ in (32, 8):
        p = torch.ones(300, device=DEV)
        m, v = dx.detox_adamw_state([p], bits=bits_)
        g = torch.ones(300, device=DEV)
        g[3], g[200], g[299] = float("nan"), float("inf"), float("-inf")
        dx.detox_adamw([p], [g], m, v, 1, 0.1)
        bad = torch.zeros(300, dtype=torch.bool, device=DEV)
        bad[[3, 200, 299]] = True
        assert bool(p[bad].isnan().all()) and bool(p[~bad].isfinite().all())
        state = [taken(m[0]), taken(v[0])] if bits_ == 8 else [m[0], v[0]]
        for s in state:
            assert bool(s[~bad].isfinite().all()) and not bool(s[bad].isfinite().any())
        assert bool((state[0][~bad] > 0.08).all())                       # and the block's scale is the finite entries'


def test_many_tensors_of_several_kinds_in_one_call():
    gen = torch.Generator(device=DEV).manual_seed(3)
    sizes = [(i * 37) % 701 + 1 for i in range(800)]
    types = [(F32, F32, False), (BF16, F32, True), (BF16, BF16, False)]
    kinds = [types[i * i % 3] for i in range(800)]
    make = lambda: ([vector(n, torch.Generator(device=DEV).manual_seed(n), 0.1, k[0]) for n, k in zip(sizes, kinds)],  # noqa: E731
                    [vector(n, torch.Generator(device=DEV).manual_seed(n + 1), 0.1) if k[2] else None for n, k in zip(sizes, kinds)])
    g = [vector(n, gen, 1e-2, k[1]) for n, k in zip(sizes, kinds)]
    for bits_ in (32, 8):
        p, w = make()
        m, v = dx.detox_adamw_state(p, bits_)
        launches = dx.kernel_launch_count()
        dx.detox_adamw(p, g, m, v, 1, 1e-2, masters=w, seed=3)
        assert dx.kernel_launch_count() - launches <= 6
        # one by one they are the same in 32 bits; in 8 bits the random bits go by the place in the list
        p1, w1 = make()
        m1, v1 = dx.detox_adamw_state(p1, bits_)
        if bits_ == 32:
            for i in range(800):
                dx.detox_adamw([p1[i]], [g[i]], [m1[i]], [v1[i]], 1, 1e-2, masters=[w1[i]])
        else:
            dx.detox_adamw(p1, g, m1, v1, 1, 1e-2, masters=w1, seed=3)
        flat = lambda xs: [t for x in xs if x is not None for t in (x if isinstance(x, tuple) else (x,))]  # noqa: E731
        for a, b in zip(flat(p + w + m + v), flat(p1 + w1 + m1 + v1)):
            assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))


def test_slices_of_one_vector_leave_what_lies_between():
    flat, state = torch.ones(10_000, device=DEV), torch.zeros((2, 10_000), device=DEV)
    spans = [(1, 130), (131, 4242), (4300, 9999)]
    cut = lambda x: [x[a:b] for a, b in spans]  # noqa: E731
    g = torch.randn(10_000, device=DEV)
    dx.detox_adamw(cut(flat), cut(g), cut(state[0]), cut(state[1]), 1, 0.1)
    between = torch.ones(10_000, dtype=torch.bool, device=DEV)
    for a, b in spans:
        between[a:b] = False
    assert bool((flat[between] == 1).all()) and bool((state[:, between] == 0).all())
    assert bool((flat[~between] != 1).all()) and bool((state[:, ~between] != 0).all())


@pytest.mark.parametrize("bits_", [32, 8])
def test_step_and_rate_from_the_device_and_a_captured_step(bits_):
    gen = torch.Generator(device=DEV).manual_seed(4)
    start, grads = [vector(5000, gen), vector(77, gen)], [[vector(5000, gen), vector(77, gen)] for _ in range(4)]
    rates = [0.1, 0.02, 0.3, 0.05]
    eager = [x.clone() for x in start]
    m, v = dx.detox_adamw_state(eager, bits_)
    want = []
    for i in range(4):
        dx.detox_adamw(eager, grads[i], m, v, i + 1, rates[i], weight_decay=0.1, seed=9)
        want.append([x.clone() for x in eager])
    p, g = [x.clone() for x in start], [x.clone() for x in grads[0]]
    m, v = dx.detox_adamw_state(p, bits_)
    step, lr = torch.zeros((), dtype=torch.int64, device=DEV), torch.zeros(1, device=DEV)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step += 1
        dx.detox_adamw(p, g, m, v, step, lr, weight_decay=0.1, seed=9)
    assert all(torch.equal(a, b) for a, b in zip(p, start))              # capturing runs nothing
    for i in range(4):
        for a, b in zip(g, grads[i]):
            a.copy_(b)
        lr.fill_(rates[i])
        graph.replay()
        # the corrections come from expm1f and sqrtf there: a few units of the step, 4 x 0.3 at most, in all steps so far; 8 bits: and a state's
        # entry on the other side where that decides (not here: the states do not depend on the corrections)
        for a, b in zip(p, want[i]):
            assert bool(((a - b).abs() <= (i + 1) * 16 * U * 4).all())
    assert int(step) == 4
    dx.detox_adamw(p, g, m, v, torch.zeros(1, dtype=torch.int64, device=DEV), 0.1)   # a step below 1 counts as the first
    assert all(bool(x.isfinite().all()) for x in p)


def test_offsets_beyond_32_bits():
    """A tensor of more than 2^31 entries: its first, its last and those around 2^31 go like a small tensor's."""
    n, k = 2 ** 31 + 9001, 4096
    gen = torch.Generator(device=DEV).manual_seed(6)
    some, grad = vector(k, gen, 0.05, BF16), vector(k, gen, 1e-2, BF16)
    p, g = torch.zeros(n, dtype=BF16, device=DEV), torch.zeros(n, dtype=BF16, device=DEV)
    places = (0, 2 ** 30 - 77, 2 ** 31 - 2049, n - k)
    for a in places:
        p[a: a + k], g[a: a + k] = some, grad
    m, v = dx.detox_adamw_state([p])
    dx.detox_adamw([p], [g], m, v, 1, 1e-2, weight_decay=0.1)
    want = some.clone()
    wm, wv = dx.detox_adamw_state([want])
    dx.detox_adamw([want], [grad], wm, wv, 1, 1e-2, weight_decay=0.1)
    for a in places:
        assert torch.equal(p[a: a + k], want) and torch.equal(m[0][a: a + k], wm[0]) and torch.equal(v[0][a: a + k], wv[0])
    assert not bool(p[k: 2 ** 30 - 77: 4099].any())


def test_refusals():
    p = torch.zeros(64, device=DEV)
    m, v = dx.detox_adamw_state([p])
    m8, v8 = dx.detox_adamw_state([p], bits=8)
    ok = lambda **k: dx.detox_adamw(**{**dict(params=[p], grads=[p + 1], m=m, v=v, step=1, lr=0.1), **k})  # noqa: E731
    ok()
    for error, bad in ((ValueError, dict(grads=[torch.zeros(65, device=DEV)])), (ValueError, dict(m=[torch.zeros(63, device=DEV)])),
                       (TypeError, dict(m=[m[0].to(BF16)])), (TypeError, dict(m=m8)), (TypeError, dict(v=v8)), (ValueError, dict(grads=[])),
                       (ValueError, dict(params=[torch.zeros((64, 2), device=DEV)[:, 0]])), (TypeError, dict(grads=[torch.zeros(64)])),
                       (TypeError, dict(params=[torch.zeros(64, dtype=torch.float64, device=DEV)])), (TypeError, dict(masters=[p.to(BF16)])),
                       (dx.DetoxError, dict(masters=[torch.zeros(64, device=DEV)])), (dx.DetoxError, dict(step=0)), (dx.DetoxError, dict(lr=float("nan"))),
                       (dx.DetoxError, dict(beta1=1.0)), (dx.DetoxError, dict(eps=0.0)), (ValueError, dict(weight_decay=[0.1, 0.1])),
                       (TypeError, dict(step=torch.ones(1, device=DEV))), (TypeError, dict(lr=torch.ones(2, device=DEV))),
                       (TypeError, dict(lr=torch.ones(1))), (ValueError, dict(m=[(m8[0][0], m8[0][1][:0])], v=v8))):
        with pytest.raises(error):
            ok(**bad)
    both = dict(grads=[p + 1, p + 1], weight_decay=[0.1, 0.0])
    other = [torch.zeros(64, device=DEV) for _ in range(3)]
    for bad in (dict(params=[p, p], m=[m[0], other[0]], v=[v[0], other[1]]), dict(params=[p, other[0]], m=[m[0], m[0]], v=[v[0], other[1]]),
                dict(params=[p, other[0]], m=[m[0], v[0]], v=[v[0], other[1]])):
        with pytest.raises(ValueError, match="twice"):
            ok(**both, **bad)
    ok(**both, params=[p, other[0]], m=[m[0], other[1]], v=[v[0], other[2]])
    w = torch.zeros(64, device=DEV, requires_grad=True)
    with pytest.raises(RuntimeError, match="requires grad"):
        ok(params=[w])
    with torch.no_grad():
        ok(params=[w])
    loss = (w * w).sum()
    with torch.no_grad():
        ok(params=[w])
    with pytest.raises(RuntimeError, match="modified"):
        loss.backward()                            # it needs the weights as they were
