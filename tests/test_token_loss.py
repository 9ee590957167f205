"""Losses over logits against 64 bits: log-probabilities of chosen tokens, the clipped policy loss, the preference loss."""
import math

import pytest
import torch

import paper_1907_12205_b200 as dx

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TYPES = [torch.bfloat16, torch.float16, torch.float32]
HALF = {t: torch.finfo(t).eps / 2 for t in TYPES}
TINY = {torch.bfloat16: 2.0 ** -134, torch.float16: 2.0 ** -25, torch.float32: 2.0 ** -126}   # (fp32: the powers flush what is smaller)
U = 2.0 ** -24
INF, NAN = float("inf"), float("nan")


def logits(rows, vocab, dtype, pad=0, offset=0, seed=0, size=3.0):
    gen = torch.Generator(device=DEV).manual_seed(seed)
    flat = (size * torch.randn(rows * (vocab + pad) + offset, generator=gen, device=DEV)).to(dtype)
    z = flat[offset:].view(rows, vocab + pad)[:, :vocab]
    y = torch.randint(0, vocab, (rows,), generator=gen, device=DEV)
    return z, y


def slack(z, scale):
    """How far a row's logp or lse may be off in fp32, and the relative error of its probabilities.  Exponents: a factor and a product rounded, twice 2^-24 of the
    row's range and of its largest entry's size; powers and logarithm: 2^-22 and a few units; sums: fewer than 100 additions one after another."""
    x = z.double() * scale
    x = torch.where(x.isinf(), torch.zeros_like(x), x)
    return U * (120 + 6 * (x.amax(1) - x.amin(1)) + 6 * x.abs().amax(1))


def exact_logp(z, y, scale):
    x = z.double() * scale
    lse = torch.logsumexp(x, 1)
    return torch.where(y < 0, 0.0, x.gather(1, y.clamp(min=0)[:, None].long())[:, 0] - lse), lse, torch.exp(x - lse[:, None])


def exact_dz(coef, p, y, scale):
    dz = -p * coef[:, None]
    dz.scatter_add_(1, y.clamp(min=0)[:, None].long(), coef[:, None])
    return torch.where((y >= 0)[:, None], dz, 0.0) * scale


def dz_bound(want, coef, coef_off, p, y, scale, dtype, off):
    """A rounding to the type; the coefficient's error; the probabilities'."""
    own = torch.zeros_like(p).scatter_(1, y.clamp(min=0)[:, None].long(), 1.0)
    near = (own - p).abs() * coef_off[:, None] + coef.abs()[:, None] * (p * off[:, None] + 4 * U * (own + p))
    return want.abs() * HALF[dtype] * 1.001 + 1.01 * scale * near + TINY[dtype]


SHAPES = [(1, 1), (3, 2), (5, 7), (9, 100), (40, 256), (33, 1000), (2, 1025), (70, 2051), (4, 4099), (300, 3001), (3, 8200), (5, 16390), (2, 32000),
          (7, 32770), (160, 5000), (80, 50257), (2, 131072), (1, 140001), (2, 262144), (2, 24584), (1, 75000), (2, 100008), (1, 120007),
          (2, 170000), (1, 200008), (1, 230000)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,vocab", SHAPES)
def test_logp_and_its_gradient(dtype, rows, vocab):
    for pad, offset, index, scale in ((0, 0, torch.int64, 1.0), (5, 3, torch.int32, 0.7)):
        z, y = logits(rows, vocab, dtype, pad, offset, seed=vocab)
        y = y.to(index)
        if rows > 2:
            y[1] = -1
        y[0] = vocab - 1
        want, lse, p = exact_logp(z, y, scale)
        off = slack(z, scale)
        got = dx.detox_token_logp(z, y, scale=scale)
        assert bool(((got.logp.double() - want).abs() <= off).all())
        assert bool(((got.lse.double() - torch.where(y < 0, 0.0, lse)).abs() <= off).all())
        d = torch.randn(rows, device=DEV, generator=torch.Generator(device=DEV).manual_seed(3))
        if rows > 4:
            d[2] = 0.0
        dz = dx.detox_token_logp_backward(d, z, y, got.lse, scale=scale)
        exact = exact_dz(d.double(), p, y, scale)
        # the rounding of lse to fp32 enters every probability
        bound = dz_bound(exact, d.double(), 2 * U * d.abs().double(), p, y, scale, dtype, 2 * off + 2 * U * lse.abs())
        assert dz.dtype == dtype and bool(((dz.double() - exact).abs() <= bound).all())
        if rows > 4:
            assert bool((dz[1:3] == 0).all())
        z2 = torch.empty_strided(z.shape, z.stride(), dtype=dtype, device=DEV).copy_(z)   # in place
        assert torch.equal(dx.detox_token_logp_backward(d, z2, y, got.lse, scale=scale, dz=z2), dz) and torch.equal(z2, dz)


LOW, HIGH, KL = 0.2, 0.3, 0.1


def policy_inputs(z, y, scale, seed=1, ref=True):
    gen = torch.Generator(device=DEV).manual_seed(seed)
    rows = z.shape[0]
    logp, _, _ = exact_logp(z, y, scale)
    gap = 0.4 * torch.randn(rows, generator=gen, device=DEV, dtype=torch.float64)
    for edge in (math.log(1 - LOW), math.log(1 + HIGH)):                 # on a border rounding decides
        gap = torch.where((gap - edge).abs() < 1e-3, gap + 5e-3, gap)
    return ((logp - gap).float(), torch.randn(rows, generator=gen, device=DEV),
            (logp + 0.5 * torch.randn(rows, generator=gen, device=DEV, dtype=torch.float64)).float() if ref else None,
            torch.rand(rows, generator=gen, device=DEV) / rows)


def exact_policy(z, y, scale, old, a, ref, w, off):
    """stats, logp, dz, and the bounds of stats and of the coefficients."""
    logp, _, p = exact_logp(z, y, scale)
    old, a, w = old.double(), a.double(), torch.where((y < 0) | (w == 0), 0.0, w.double())
    r = torch.exp(logp - old)
    held = r.clamp(1 - LOW, 1 + HIGH)
    clipped = r * a > held * a
    pg = -torch.minimum(r * a, held * a)
    slope = torch.where(clipped, 0.0, -r * a)
    d = torch.zeros_like(r) if ref is None else ref.double() - logp
    kl, slope = torch.exp(d) - d - 1, slope - KL * (torch.exp(d) - 1)
    kl, slope, pg = (torch.where(w == 0, 0.0, x) for x in (kl, slope, pg))
    stats = torch.stack([(w * (pg + KL * kl)).sum(), (w * pg).sum(), (w * kl).sum(), (w * clipped).sum()])
    # __expf is off by 2 units and one for each 1 / 1.17 of its argument; four more roundings
    unit = off + U * (16 + 8 * (logp - old).abs() + 8 * d.abs())
    slope_off = r * a.abs() * unit + KL * (torch.exp(d) + 1) * unit
    kl_off = (torch.exp(d) + 1) * unit
    each = torch.stack([w * (r * a.abs() * unit + KL * kl_off), w * r * a.abs() * unit, w * kl_off, 4 * U * w]).abs()
    values = torch.stack([w * (pg.abs() + KL * kl), w * pg.abs(), w * kl, w]).abs()
    each, values = (torch.where(w == 0, 0.0, x) for x in (each, values))
    return stats, torch.where(w == 0, 0.0, logp), w * slope, p, (each + 4 * U * values).sum(1) + U * stats.abs(), w.abs() * slope_off


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,vocab", SHAPES)
def test_policy_loss(dtype, rows, vocab):
    for pad, offset, scale, ref in ((0, 0, 1.0, True), (5, 1, 1.25, False)):
        z, y = logits(rows, vocab, dtype, pad, offset, seed=rows + vocab)
        if rows > 4:
            y[1] = -1
        old, a, reference, w = policy_inputs(z, y, scale, ref=ref)
        if rows > 4:
            w[3] = 0.0
        off = slack(z, scale)
        stats, logp, coef, p, stats_off, coef_off = exact_policy(z, y, scale, old, a, reference, w, off)
        got = dx.detox_policy_loss(z, y, old, a, reference, w, LOW, HIGH, KL, scale, grad_scale=4.0)
        assert bool(((got.stats.double() - stats).abs() <= stats_off).all()), (got.stats.double() - stats, stats_off)
        assert bool(((got.logp.double() - logp).abs() <= off).all())
        exact = exact_dz(4.0 * coef, p, y, scale)
        bound = dz_bound(exact, 4.0 * coef, 4.0 * coef_off + 8 * U * coef.abs(), p, y, scale, dtype, 2 * off)
        assert got.dz.dtype == dtype and bool(((got.dz.double() - exact).abs() <= bound).all())
        if rows > 4:
            assert bool((got.dz[[1, 3]] == 0).all())
        alone = dx.detox_policy_loss(z, y, old, a, reference, w, LOW, HIGH, KL, scale, want_grad=False)
        assert alone.dz is None and torch.equal(alone.stats, got.stats) and torch.equal(alone.logp, got.logp)
        z2 = torch.empty_strided(z.shape, z.stride(), dtype=dtype, device=DEV).copy_(z)
        here = dx.detox_policy_loss(z2, y, old, a, reference, w, LOW, HIGH, KL, scale, grad_scale=4.0, dz=z2)
        assert torch.equal(z2, got.dz) and torch.equal(here.stats, got.stats)


@pytest.mark.parametrize("vocab", [37, 3000, 40000])
def test_policy_loss_without_weights_and_with_rows_enough_for_several_turns(vocab):
    rows = 2000
    z, y = logits(rows, vocab, torch.bfloat16, seed=4)
    y[torch.rand(rows, device=DEV, generator=torch.Generator(device=DEV).manual_seed(1)) < 0.4] = -1
    y[100:700] = -1
    old, a, ref, _ = policy_inputs(z, y, 1.0)
    w = torch.full((rows,), 1.0 / rows, device=DEV)
    off = slack(z, 1.0)
    stats, logp, coef, p, stats_off, coef_off = exact_policy(z, y, 1.0, old, a, ref, w, off)
    got = dx.detox_policy_loss(z, y, old, a, ref, clip_low=LOW, clip_high=HIGH, kl_coef=KL)
    assert bool(((got.stats.double() - stats).abs() <= stats_off + U * stats.abs()).all())
    exact = exact_dz(coef, p, y, 1.0)
    bound = dz_bound(exact, coef, coef_off + 8 * U * coef.abs(), p, y, 1.0, torch.bfloat16, 2 * off)
    assert bool(((got.dz.double() - exact).abs() <= bound).all())
    again = dx.detox_policy_loss(z, y, old, a, ref, clip_low=LOW, clip_high=HIGH, kl_coef=KL)
    assert torch.equal(again.stats, got.stats) and torch.equal(again.dz, got.dz)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("vocab", [5, 300, 5000, 70000])
def test_masked_entries_empty_rows_and_nan(dtype, vocab):
    z, y = logits(8, vocab, dtype, seed=2)
    y[:] = 1
    z[0, 2:] = -INF                                # masked entries
    z[1] = -INF                                    # nothing left
    z[2] = NAN                                     # no chosen token there: not looked at
    y[2] = -1
    z[3, vocab - 1] = NAN
    z[4, 0] = INF
    z[5] = torch.finfo(dtype).min                  # a mask of the lowest value: every entry alike
    y[6] = vocab                                   # outside the vocabulary
    z[7, 0] = -INF
    ones = torch.ones(8, device=DEV)
    got = dx.detox_token_logp(z, y)
    dz = dx.detox_token_logp_backward(ones, z, y, got.lse)
    pol = dx.detox_policy_loss(z, y, torch.zeros(8, device=DEV), ones, weight=ones)
    exact = torch.log_softmax(z.double(), 1)
    for logp in (got.logp, pol.logp):
        assert abs(float(logp[0] - exact[0, 1])) <= 200 * U and abs(float(logp[7] - exact[7, 1])) <= 300 * U
        assert float(logp[1]) == -INF and float(logp[2]) == 0.0
        assert bool(logp[[3, 4, 6]].isnan().all())
        # -65504 is a number like others; -3.4e38 (bf16 and fp32) times log2(e) is not a number of fp32: such a row counts as empty
        assert abs(float(logp[5]) + math.log(vocab)) <= 200 * U if dtype == torch.float16 else float(logp[5]) == -INF
    assert float(got.lse[1]) == -INF and bool(pol.stats[:1].isnan())
    for g in (dz, pol.dz):
        if dtype != torch.float16:
            assert bool((g[5] == 0).all())
        assert bool((g[0, 2:] == 0).all()) and bool((g[1:3] == 0).all()) and bool((g[7, 0] == 0).all())
        assert bool(g[6].isnan().all()) and bool(g[3].isnan().any()) and bool(g[4].isnan().any())
        assert abs(float(g[0].double().sum())) <= 4 * HALF[dtype]        # probabilities add up to one


def test_reference_probabilities_far_from_the_policys():
    """The KL term's slope is kl_coef (1 - exp(ref - logp)): kl_coef itself where the reference gives nothing, however far its logarithm lies."""
    z, y = logits(6, 90, torch.float32)
    z, y = z[:1].expand(6, 90).contiguous(), y[:1].expand(6).contiguous()
    old = dx.detox_token_logp(z, y).logp
    ref = old + torch.tensor([0.0, -100.0, -1e6, -INF, 3.0, 60.0], device=DEV)
    one = torch.ones(6, device=DEV)
    got = dx.detox_policy_loss(z, y, old, 0 * one, ref, one, kl_coef=0.5)
    own = torch.exp(old[0].double())
    # with advantage 0 only that slope is left: dz at the chosen token is slope (1 - p)
    slope = got.dz[torch.arange(6, device=DEV), y].double() / (1 - own)
    want = 0.5 * (1 - torch.exp(ref.double() - old.double()))
    assert bool(((slope - want).abs() <= 600 * U * (want.abs() + 1)).all()), (slope, want)
    assert float(got.kl) == INF and float(got.pg) == 0.0
    none = dx.detox_policy_loss(z[:3], y[:3], old[:3], 0 * one[:3], ref[:3], one[:3], kl_coef=0.5)
    exact = (torch.exp(ref.double() - old.double()) - 1 - (ref.double() - old.double()))[:3].sum()
    assert abs(float(none.kl) - float(exact)) <= 8 * U * float(exact)
    z[0, y[0]] = -INF                              # a chosen token that the policy gives nothing
    gone = dx.detox_policy_loss(z[:1], y[:1], old[:1], one[:1], old[:1], one[:1], kl_coef=0.5)
    assert float(gone.logp) == -INF and float(gone.kl) == INF


def test_rows_of_weight_zero_are_not_looked_at():
    z, y = logits(6, 500, torch.bfloat16)
    old, a, ref, w = policy_inputs(z, y, 1.0)
    want = dx.detox_policy_loss(z[:4], y[:4], old[:4], a[:4], ref[:4], w[:4])
    z, old, a, ref = z.clone(), old.clone(), a.clone(), ref.clone()
    z[4:], old[4:], a[4:], ref[4:] = NAN, INF, NAN, -INF
    w[4] = 0.0
    y[5] = -7
    got = dx.detox_policy_loss(z, y, old, a, ref, w)
    assert torch.equal(got.stats, want.stats) and torch.equal(got.dz[:4], want.dz) and bool((got.dz[4:] == 0).all())


def preference(z, y, offsets, ref, beta, smoothing, scale):
    logp, _, p = exact_logp(z, y, scale)
    sums = torch.stack([logp[a:b].sum() for a, b in zip(offsets, offsets[1:])]) if len(offsets) > 1 else logp.new_zeros(0)
    lead = (sums - ref.double()).view(-1, 2)
    h = beta * (lead[:, 0] - lead[:, 1])
    sig = torch.nn.functional.logsigmoid
    loss = (-(1 - smoothing) * sig(h) - smoothing * sig(-h)).mean()
    dh = (smoothing * torch.sigmoid(h) - (1 - smoothing) * torch.sigmoid(-h)) * beta / h.numel()
    coef = torch.zeros_like(logp)
    for i, (a, b) in enumerate(zip(offsets, offsets[1:])):
        coef[a:b] = dh[i // 2] * (1 - 2 * (i % 2))
    return loss, h, sums, torch.where(y < 0, 0.0, coef), p


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("lengths,behind,vocab", [([1, 1], 0, 40), ([3, 0], 2, 129), ([0, 0], 3, 20), ([40, 300, 7, 1], 9, 1001),
                                                  ([700, 513, 0, 90, 33, 34], 1, 257), ([20, 15], 0, 33000)])
def test_preference_loss(dtype, lengths, behind, vocab):
    rows = sum(lengths) + behind
    for pad, scale, smoothing in ((0, 1.0, 0.0), (3, 0.8, 0.2)):
        z, y = logits(rows, vocab, dtype, pad, seed=rows)
        y[torch.rand(rows, device=DEV, generator=torch.Generator(device=DEV).manual_seed(1)) < 0.3] = -1
        offsets = [0] + torch.tensor(lengths).cumsum(0).tolist()
        plain = preference(z, y, offsets, torch.zeros(len(lengths), device=DEV), 0.1, 0.0, scale)[2]
        ref = (plain + 4.0 * torch.randn(len(lengths), device=DEV, generator=torch.Generator(device=DEV).manual_seed(2))).float()
        loss, h, sums, coef, p = preference(z, y, offsets, ref, 0.3, smoothing, scale)
        off = torch.where(y < 0, 0.0, slack(z, scale))
        sums_off = torch.stack([off[a:b].sum() for a, b in zip(offsets, offsets[1:])])
        h_off = 0.3 * sums_off.view(-1, 2).sum(1) + 2 * U * h.abs()
        got = dx.detox_preference_loss(z, y, torch.tensor(offsets, dtype=torch.int32, device=DEV), ref, beta=0.3, smoothing=smoothing, scale=scale,
                                       grad_scale=2.0)
        assert bool(((got.sums.double() - sums).abs() <= sums_off + U * sums.abs()).all())
        assert bool(((got.margin.double() - h).abs() <= h_off).all())
        # log(1 + e^-|h|) and the sum: six roundings of numbers up to |h| + 1
        assert abs(float(got.loss.double()[0] - loss)) <= float((h_off + 12 * U * (1 + h.abs())).mean())
        # the sigmoid's slope is at most 1 / 4; expf, a division and three products
        off_h = torch.zeros(rows, dtype=torch.float64, device=DEV)
        for i, (a, b) in enumerate(zip(offsets, offsets[1:])):
            off_h[a:b] = 0.3 / h.numel() * h_off[i // 2] / 4
        exact = exact_dz(2.0 * coef, p, y, scale)
        bound = dz_bound(exact, 2.0 * coef, 2.0 * (off_h + 24 * U * coef.abs()), p, y, scale, dtype, 2 * slack(z, scale) + 8 * U * torch.logsumexp(z.double() * scale, 1).abs())
        assert bool(((got.dz.double() - exact).abs() <= bound).all())
        assert bool((got.dz[sum(lengths):] == 0).all())
        alone = dx.detox_preference_loss(z, y, torch.tensor(offsets, dtype=torch.int32, device=DEV), ref, beta=0.3, smoothing=smoothing, scale=scale,
                                         want_grad=False)
        assert alone.dz is None and torch.equal(alone.loss, got.loss) and torch.equal(alone.margin, got.margin)


def test_preference_loss_of_very_different_answers_and_of_many_pairs():
    z, y = logits(4, 50, torch.float32)
    ref = torch.tensor([1e4, -1e4, -3e38, 3e38], device=DEV)
    got = dx.detox_preference_loss(z, y, torch.tensor([0, 1, 2, 3, 4], dtype=torch.int32, device=DEV), ref, beta=1.0)
    assert float(got.margin[0]) < -1e4 and float(got.margin[1]) == INF and abs(float(got.loss) - float(-got.margin[0]) / 2) <= 4
    assert bool((got.dz[2:] == 0).all()) and bool(got.dz.isfinite().all())
    pairs = 3000                                   # more than CTAs
    z, y = logits(2 * pairs + 1, 33, torch.bfloat16)
    offsets = torch.arange(2 * pairs + 1, dtype=torch.int32, device=DEV)
    ref = torch.randn(2 * pairs, device=DEV, generator=torch.Generator(device=DEV).manual_seed(0)) - 4
    loss, h, _, coef, p = preference(z, y, offsets.tolist(), ref, 0.5, 0.1, 1.0)
    got = dx.detox_preference_loss(z, y, offsets, ref, beta=0.5, smoothing=0.1)
    off = float(slack(z, 1.0).max())
    assert bool(((got.margin.double() - h).abs() <= 2 * off + 2 * U * h.abs()).all()) and abs(float(got.loss) - float(loss)) <= 2 * off + 24 * U * 8
    exact = exact_dz(coef, p, y, 1.0)
    assert bool(((got.dz.double() - exact).abs() <= HALF[torch.bfloat16] * exact.abs() * 1.001 + 8 * off * coef.abs()[:, None] + TINY[torch.bfloat16]).all())


def test_offsets_out_of_range_are_clamped():
    z, y = logits(6, 40, torch.float32)
    for bad in ([0, 3, 100], [-5, 2, 6], [4, 1, 3], [2 ** 31 - 1, -2 ** 31, 5], [7, 7, 7]):
        got = dx.detox_preference_loss(z, y, torch.tensor(bad, dtype=torch.int32, device=DEV), torch.zeros(2, device=DEV))
        assert bool(got.dz.isfinite().all()) and bool(got.sums.isfinite().all())
    none = dx.detox_preference_loss(z, y, torch.zeros(1, dtype=torch.int32, device=DEV), torch.empty(0, device=DEV))
    assert float(none.loss) == 0.0 and bool((none.dz == 0).all()) and none.margin.shape == (0,)


def test_no_rows():
    z, y, f = torch.empty((0, 40), device=DEV), torch.empty(0, dtype=torch.int64, device=DEV), torch.empty(0, device=DEV)
    assert dx.detox_token_logp(z, y).logp.shape == (0,)
    assert dx.detox_token_logp_backward(f, z, y, f).shape == (0, 40)
    got = dx.detox_policy_loss(z, y, f, f)
    assert bool((got.stats == 0).all()) and got.dz.shape == (0, 40)
    got = dx.detox_preference_loss(z, y, torch.zeros(3, dtype=torch.int32, device=DEV), torch.zeros(2, device=DEV))
    assert abs(float(got.loss) - math.log(2)) <= 4 * U and got.dz.shape == (0, 40)


def test_gradients_against_differences():
    """Along a random direction: (f(z + h) - f(z - h)) / 2h is off by h^2 / 6 of the third derivative (below 10 here) and the losses' rounding over h."""
    rows, vocab, h = 24, 60, 2.0 ** -7
    z, y = logits(rows, vocab, torch.float32, size=1.0)
    old, a, ref, w = policy_inputs(z, y, 1.0)
    off = torch.tensor([0, 5, 9, 17, 24], dtype=torch.int32, device=DEV)
    sums = torch.randn(4, device=DEV, generator=torch.Generator(device=DEV).manual_seed(8)) * 3 - 20

    def logp(x, grad=False):
        got = dx.detox_token_logp(x, y)
        return dx.detox_token_logp_backward(w, x, y, got.lse) if grad else float((got.logp.double() * w.double()).sum())

    def policy(x, grad=False):
        got = dx.detox_policy_loss(x, y, old, a, ref, w, LOW, HIGH, KL)
        return got.dz if grad else float(got.loss)

    def pairs(x, grad=False):
        got = dx.detox_preference_loss(x, y, off, sums, beta=0.2, smoothing=0.1)
        return got.dz if grad else float(got.loss)

    for f in (logp, policy, pairs):
        grad = f(z, True).double()
        for seed in range(3):
            d = torch.randn(z.shape, device=DEV, generator=torch.Generator(device=DEV).manual_seed(seed))
            d /= d.norm()
            diff = (f(z + h * d) - f(z - h * d)) / (2 * h)
            assert abs(diff - float((grad * d.double()).sum())) <= 10 * h * h / 6 + 400 * U / h


def test_outside_and_behind_nothing_is_written():
    rows, vocab = 21, 1003
    z, y = logits(rows, vocab, torch.bfloat16, pad=5, offset=1)
    old, a, ref, w = policy_inputs(z, y, 1.0)
    size = dx.detox_policy_loss_workspace_bytes(rows)
    ws = torch.full((size + 512,), 0x5A, dtype=torch.uint8, device=DEV)
    buffer = torch.full((rows + 2, vocab + 9), 7.0, dtype=torch.bfloat16, device=DEV)
    dx.detox_policy_loss(z, y, old, a, ref, w, dz=buffer[1:-1, :vocab], ws=ws[256:256 + size])
    assert bool((buffer[[0, -1]] == 7).all()) and bool((buffer[:, vocab:] == 7).all())
    assert bool((ws[:256] == 0x5A).all()) and bool((ws[256 + size:] == 0x5A).all())
    size = dx.detox_preference_loss_workspace_bytes(rows, 1)
    ws = torch.full((size + 512,), 0x5A, dtype=torch.uint8, device=DEV)
    buffer.fill_(7.0)
    dx.detox_preference_loss(z, y, torch.tensor([0, 9, 20], dtype=torch.int32, device=DEV), torch.zeros(2, device=DEV), dz=buffer[1:-1, :vocab],
                             ws=ws[256:256 + size])
    assert bool((buffer[[0, -1]] == 7).all()) and bool((buffer[:, vocab:] == 7).all()) and bool((buffer[-2, :vocab] == 0).all())
    assert bool((ws[:256] == 0x5A).all()) and bool((ws[256 + size:] == 0x5A).all())


def test_offsets_beyond_32_bits():
    """Logits of more than 2^31 entries, the last rows of them chosen."""
    rows, vocab = 8200, 262144
    z = torch.empty((rows, vocab), dtype=torch.bfloat16, device=DEV)
    part, _ = logits(4, vocab, torch.bfloat16)
    z[-4:] = part
    y = torch.full((rows,), -1, dtype=torch.int32, device=DEV)
    y[-4:] = torch.tensor([0, 5, vocab - 1, 77], device=DEV)
    old, a, _, _ = policy_inputs(part, y[-4:], 1.0)
    w = torch.full((4,), 0.25, device=DEV)
    want = dx.detox_policy_loss(part, y[-4:], old, a, weight=w)
    score = dx.detox_token_logp(part, y[-4:])
    assert torch.equal(dx.detox_token_logp(z, y).logp[-4:], score.logp)
    far = lambda x: torch.cat([torch.zeros(rows - 4, device=DEV), x])  # noqa: E731
    back = dx.detox_token_logp_backward(far(w), z, y, far(score.lse))
    assert torch.equal(back[-4:], dx.detox_token_logp_backward(w, part, y[-4:], score.lse)) and bool((back[1:8000:501] == 0).all())
    got = dx.detox_policy_loss(z, y, far(old), far(a), weight=far(w), dz=z)
    # (clusters of another size, another order of the sums)
    assert bool(((got.dz[-4:].double() - want.dz.double()).abs() <= 2.02 * HALF[torch.bfloat16] * want.dz.double().abs() + 1e-30).all())
    assert bool((z[1:8000:501] == 0).all()) and bool(((got.stats - want.stats).abs() <= 64 * U).all())
