"""The worker-side operators against their definitions in 64 bits: the 8-bit form of kept activations, the root-mean-square
norm, the gated pair of projections, and the backward passes.

Where inputs are small whole numbers every sum is exact in fp32, and the outputs have to be the rounded exact values.
Elsewhere the bounds are the worst case of the arithmetic, entry by entry: an fp32 sum of n terms is off by at most
n 2^-23 times the sum of their absolute values (each addition may truncate), and a rounding to a type by its half-unit
(2^-8 of the value in bf16, 2^-11 in fp16, 2^-24 in fp32)."""
import math

import numpy as np
import pytest
import torch

import paper_1907_12205_b200 as dx

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16
HALF_UNIT = {F32: 2.0 ** -24, F16: 2.0 ** -11, BF16: 2.0 ** -8}    # 24, 11 and 8 significant bits
TINY = {F32: 2.0 ** -149, F16: 2.0 ** -25, BF16: 2.0 ** -134}   # half the smallest step
ACTS = {"silu": dx.ACT_SILU, "gelu": dx.ACT_GELU, "relu": dx.ACT_RELU}


def strided(t, pad, shift=0):
    """The same values in rows `pad` entries further apart, starting `shift` entries into the buffer."""
    rows, cols = t.shape
    flat = torch.full((rows * (cols + pad) + shift + 8,), float("nan"), dtype=t.dtype, device=t.device)
    v = flat[shift: shift + rows * (cols + pad)].view(rows, cols + pad)[:, :cols]
    v.copy_(t)
    return v


def randn(gen, *shape, scale=1.0):
    return torch.randn(shape, generator=gen, dtype=torch.float64) * scale


def ints(gen, lo, hi, *shape):
    return torch.randint(lo, hi + 1, shape, generator=gen).double()


def generator(seed):
    return torch.Generator().manual_seed(seed)


def within(got, ref, bound, what):
    got = got.detach().cpu().double()
    assert got.shape == ref.shape
    bad = ~((got - ref).abs() <= bound)
    assert not bad.any(), f"{what}: {int(bad.sum())} of {bad.numel()} off, worst {float(((got - ref).abs() / bound).max())} bounds"


# ------------------------------------------------------------------------------------- the 8-bit form

def exponents(x):
    """Biased exponents by the definition, from the finite entries (64-bit numpy)."""
    rows, cols = x.shape
    out = np.empty((rows, -(-cols // 128)), np.int64)
    for b in range(out.shape[1]):
        part = np.abs(x[:, b * 128:(b + 1) * 128])
        part = np.where(np.isfinite(part), part, 0.0).max(1)
        for r, a in enumerate(part):
            e = -126
            while a > 448.0 * 2.0 ** e:
                e += 1
            out[r, b] = e + 127
    return out


def e4m3(v):
    """The e4m3 number nearest to v (ties to even), |v| <= 448; NaN and Inf become NaN."""
    v = np.asarray(v, np.float64)
    fine = np.isfinite(v)
    w = np.where(fine, v, 0.0)
    step = 2.0 ** (np.floor(np.log2(np.maximum(np.abs(w), 2.0 ** -6))) - 3)
    return np.where(fine, np.round(w / step) * step, np.nan)


def kept_by_definition(x):
    e = exponents(x)
    scale = 2.0 ** (e - 127.0)
    wide = np.repeat(scale, 128, axis=1)[:, : x.shape[1]]
    return e4m3(x / wide), e, wide


def special_rows(dtype, cols):
    """Rows of the values where a scale or a rounding can go wrong."""
    top = torch.finfo(dtype).max
    tiny = torch.finfo(dtype).smallest_normal
    gen = generator(cols)
    rows = [torch.zeros(cols, dtype=torch.float64), torch.full((cols,), top, dtype=torch.float64),
            torch.full((cols,), tiny / 4, dtype=torch.float64), torch.full((cols,), 448.0, dtype=torch.float64),
            torch.full((cols,), 449.0, dtype=torch.float64), -0.0 * torch.ones(cols, dtype=torch.float64),
            randn(gen, cols), randn(gen, cols)]
    for at, v in ((0, math.inf), (cols // 2, -math.inf), (cols - 1, math.nan)):
        rows[6][at] = v
    rows[7] *= torch.exp2(torch.randint(-20, 8, (cols,), generator=gen).double())
    return torch.stack(rows).to(dtype)


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("cols,pad,shift", [(1, 0, 0), (15, 1, 0), (16, 0, 0), (127, 1, 0), (128, 0, 0), (129, 7, 1), (300, 4, 0), (1003, 5, 3), (1024, 0, 8)])
def test_eight_bit_form_is_the_definition_bit_for_bit(dtype, cols, pad, shift):
    x = special_rows(dtype, cols)
    q, e = dx.detox_checkpoint_pack(strided(x.to(DEV), pad, shift))
    ref_q, ref_e, wide = kept_by_definition(x.double().numpy())
    assert np.array_equal(e.view(torch.uint8).cpu().numpy(), ref_e)
    got = q.float().cpu().numpy().astype(np.float64)
    assert np.array_equal(np.isnan(got), np.isnan(ref_q)) and np.array_equal(np.nan_to_num(got), np.nan_to_num(ref_q))
    for back in (F32, F16, BF16):
        out = torch.full((x.shape[0], cols + pad), 7.0, dtype=back, device=DEV)
        dx.detox_checkpoint_unpack(q, e, out=out[:, :cols])
        want = torch.from_numpy(np.nan_to_num(ref_q * wide, nan=math.nan))
        if back == F16:
            want = want.clamp(-65504, 65504)
        want = want.to(back)
        assert torch.equal(torch.isnan(out[:, :cols].cpu()), torch.isnan(want))
        assert torch.equal(torch.nan_to_num(out[:, :cols].cpu()), torch.nan_to_num(want))
        assert bool((out[:, cols:] == 7.0).all())


def test_packing_into_strided_buffers_leaves_their_padding_alone():
    x = randn(generator(3), 37, 200).to(BF16).to(DEV)
    for pad in (0, 5, 8):
        qb = torch.full((37, 200 + pad), 9, dtype=torch.uint8, device=DEV).view(torch.float8_e4m3fn)
        eb = torch.full((37, 5), 9, dtype=torch.uint8, device=DEV).view(torch.float8_e8m0fnu)
        dx.detox_checkpoint_pack(x, out=(qb[:, :200], eb[:, :2]))
        q, e = dx.detox_checkpoint_pack(x)
        assert torch.equal(qb[:, :200].view(torch.uint8), q.view(torch.uint8)) and torch.equal(eb[:, :2].view(torch.uint8), e.view(torch.uint8))
        assert bool((qb.view(torch.uint8)[:, 200:] == 9).all()) and bool((eb.view(torch.uint8)[:, 2:] == 9).all())


def test_a_checkpoint_whose_offsets_pass_32_bits():
    rows, cols = 4200, 1_048_576 + 16          # 4.4e9 entries
    x = torch.zeros((rows, cols), dtype=torch.float8_e4m3fn, device=DEV)
    e = torch.full((rows, -(-cols // 128)), 127, dtype=torch.uint8, device=DEV).view(torch.float8_e8m0fnu)
    x.view(torch.uint8)[rows - 1, cols - 3] = 0x38       # 1.0
    e.view(torch.uint8)[rows - 1, -1] = 130              # times 8
    out = dx.detox_checkpoint_unpack(x, e, BF16)
    assert float(out[rows - 1, cols - 3]) == 8.0 and float(out[-1].double().sum()) == 8.0 and float(out[: rows - 1].abs().max()) == 0.0
    q, e2 = dx.detox_checkpoint_pack(out)
    assert int(e2.view(torch.uint8)[rows - 1, -1]) == 127 + 3 - 8 and float(q[rows - 1, cols - 3].float()) == 256.0
    assert int(e2.view(torch.uint8)[: rows - 1].max()) == 1


# ------------------------------------------------------------------------------------- the norm

NORM_SHAPES = [(1, 1), (1, 2048), (3, 7), (9, 64), (17, 255), (8, 256), (5, 1000), (33, 1024), (4, 1025), (7, 2048), (3, 4100), (2, 9001), (2, 32768)]


def norm_reference(x, r, w, eps):
    s = x if r is None else x + r
    rstd = 1.0 / torch.sqrt((s * s).mean(1) + eps)
    return s, rstd, s * rstd[:, None] * w


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("rows,cols", NORM_SHAPES)
def test_norm(dtype, rows, cols):
    gen = generator(rows * 100003 + cols)
    for residual, pad, shift in ((True, 0, 0), (False, 3, 1), (True, 8, 8)):
        x = (randn(gen, rows, cols) * torch.exp(randn(gen, rows, 1))).to(dtype)
        r = randn(gen, rows, cols).to(dtype) if residual else None
        w = (1 + 0.3 * randn(gen, cols)).to(dtype)
        s, rstd, y = norm_reference(x.double(), None if r is None else r.double(), w.double(), 1e-6)
        got = dx.detox_rmsnorm(strided(x.to(DEV), pad, shift), w.to(DEV), None if r is None else strided(r.to(DEV), pad, shift),
                               eps=1e-6, want_y=True, want_q=True)
        # x + r rounds once (2^-24 of |x| + |r|), squares and their sum (positive terms: at most 64 additions in a chain
        # of registers, shuffles and warps) relatively by 2^-24 each, rsqrt by 2 units
        off = 80 * 2.0 ** -24
        cancel = 0 if r is None else (x.double().abs() + r.double().abs()) * 2.0 ** -24
        rel = off + (0 if r is None else float((cancel.square().sum(1).sqrt() / s.square().sum(1).sqrt().clamp(min=1e-300)).max()))
        within(got.rstd, rstd, rel * rstd, "rstd")
        if residual:
            within(got.sum, s, HALF_UNIT[dtype] * s.abs() + cancel + TINY[dtype], "sum")
        else:
            assert got.sum is None
        slack = (rel + 4 * 2.0 ** -24) * y.abs() + cancel * (rstd[:, None] * w.double().abs())
        within(got.y, y, HALF_UNIT[dtype] * (y.abs() + slack) + slack + TINY[dtype], "y")
        # the 8-bit form: scales by the definition unless a block's largest entry is within the slack of a boundary
        e = exponents(y.numpy())
        lo, hi = exponents((y.abs() - slack).clamp(min=0).numpy()), exponents((y.abs() + slack).numpy())
        ge = got.e.view(torch.uint8).cpu().numpy().astype(np.int64)
        assert ((ge >= lo) & (ge <= hi)).all() and (ge == e).mean() > 0.99
        scale = torch.from_numpy(np.repeat(2.0 ** (ge - 127.0), 128, axis=1)[:, :cols])
        within(got.q.float().cpu().double() * scale, y, 2.0 ** -4 * (y.abs() + slack) + 2.0 ** -10 * scale + slack, "q")


def test_norm_outputs_can_be_asked_for_one_by_one_and_in_place():
    gen = generator(5)
    x, r = randn(gen, 50, 777).to(F16).to(DEV), randn(gen, 50, 777).to(F16).to(DEV)
    w = randn(gen, 777).to(F16).to(DEV)
    full = dx.detox_rmsnorm(x, w, r, want_q=True)
    only_q = dx.detox_rmsnorm(x, w, r, want_y=False, want_q=True)
    assert only_q.y is None and torch.equal(only_q.q.view(torch.uint8), full.q.view(torch.uint8))
    only_r = dx.detox_rmsnorm(x, w, want_y=False)
    assert only_r.y is None and only_r.q is None and only_r.sum is None and only_r.rstd.shape == (50,)
    for wide in (777, 784):
        a, b = (strided(t, wide - 777) for t in (x, r))
        got = dx.detox_rmsnorm(a, w, b, sum_out=b)
        assert got.sum is b and torch.equal(b, full.sum) and torch.equal(got.y, full.y)


def test_norm_rows_do_not_meet():
    """A row of NaN, of Inf or of zeros changes no other row."""
    gen = generator(6)
    x, w = randn(gen, 6, 500).to(BF16).to(DEV), randn(gen, 500).to(BF16).to(DEV)
    clean = dx.detox_rmsnorm(x, w, want_q=True)
    y = x.clone()
    y[1] = math.nan
    y[3, 77] = math.inf
    y[4] = 0.0
    got = dx.detox_rmsnorm(y, w, want_q=True)
    for k in (0, 2, 5):
        assert torch.equal(got.y[k], clean.y[k]) and torch.equal(got.q[k].view(torch.uint8), clean.q[k].view(torch.uint8))
    assert bool(got.y[1].isnan().all()) and bool((got.y[4] == 0).all()) and abs(float(got.rstd[4]) - 1e3) < 1e-2
    assert float(got.rstd[3]) == 0.0 and bool(got.y[3, 77].isnan())


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("rows,cols", NORM_SHAPES + [(700, 96), (1500, 2050)])
def test_norm_backward(dtype, rows, cols):
    gen = generator(rows + 7 * cols)
    for extra, pad, shift in ((True, 0, 0), (False, 5, 1)):
        s, dy = randn(gen, rows, cols).to(dtype), randn(gen, rows, cols).to(dtype)
        ds = randn(gen, rows, cols).to(dtype) if extra else None
        w = (1 + 0.3 * randn(gen, cols)).to(dtype)
        rstd = (1.0 / torch.sqrt((s.double() ** 2).mean(1) + 1e-6)).float()
        gx, gw = dx.detox_rmsnorm_backward(strided(dy.to(DEV), pad, shift), strided(s.to(DEV), pad, shift), w.to(DEV), rstd.to(DEV),
                                           ds=None if ds is None else strided(ds.to(DEV), pad, shift))
        S, DY, W, R = s.double(), dy.double(), w.double(), rstd.double()[:, None]
        hat = S * R
        dot = (W * DY * hat).mean(1, keepdim=True)
        ref = R * (W * DY - hat * dot)
        size = R * ((W * DY).abs() + hat.abs() * (W * DY * hat).abs().mean(1, keepdim=True))
        if ds is not None:
            ref = ref + ds.double()
            size = size + ds.double().abs()
        # the mean of cols terms: at most 80 additions in a chain; a handful of roundings around it
        within(gx, ref, 96 * 2.0 ** -24 * size + HALF_UNIT[dtype] * (ref.abs() + size * 1e-5) + TINY[dtype], "dx")
        # dw: rows are added one after another within a CTA, then the CTAs' sums
        within(gw, (DY * hat).sum(0), (rows + 40) * 2.0 ** -24 * (DY * hat).abs().sum(0) + 1e-30, "dw")


def test_norm_backward_against_differences():
    gen = generator(11)
    rows, cols = 6, 333
    x, r = randn(gen, rows, cols).float(), randn(gen, rows, cols).float()
    w, dy, ds = (1 + 0.3 * randn(gen, cols)).float(), randn(gen, rows, cols).float(), randn(gen, rows, cols).float()
    f = dx.detox_rmsnorm(x.to(DEV), w.to(DEV), r.to(DEV))
    gx, gw = dx.detox_rmsnorm_backward(dy.to(DEV), f.sum, w.to(DEV), f.rstd, ds=ds.to(DEV))

    def loss(x, w):
        s, _, y = norm_reference(x, r.double(), w, 1e-6)
        return float((dy.double() * y).sum() + (ds.double() * s).sum())

    h = 1e-5
    for _ in range(4):
        vx, vw = randn(gen, rows, cols), randn(gen, cols)
        for got, d, name in ((gx, (vx, 0.0), "x"), (gw, (0.0, vw), "w")):
            diff = (loss(x.double() + h * d[0], w.double() + h * d[1]) - loss(x.double() - h * d[0], w.double() - h * d[1])) / (2 * h)
            along = float((got.cpu().double() * (vx if name == "x" else vw)).sum())
            # differences are off by h^2 times a third derivative of order rows * cols, fp32 by 1e-6 of the terms
            assert abs(along - diff) <= 1e-5 * math.sqrt(rows * cols) * 10, (name, along, diff)


def test_norm_backward_in_place_and_without_rows():
    gen = generator(12)
    s, dy, ds = (randn(gen, 40, 512).to(BF16).to(DEV) for _ in range(3))
    w = randn(gen, 512).to(BF16).to(DEV)
    rstd = torch.rsqrt(s.float().square().mean(1) + 1e-6)
    gx, gw = dx.detox_rmsnorm_backward(dy, s, w, rstd, ds=ds)
    for buf in (dy.clone(), ds.clone()):
        a, b = (buf, ds) if torch.equal(buf, dy) else (dy, buf)
        got, _ = dx.detox_rmsnorm_backward(a, s, w, rstd, ds=b, dx=buf)
        assert got is buf and torch.equal(buf, gx)
    e = torch.empty((0, 512), dtype=BF16, device=DEV)
    gx, gw = dx.detox_rmsnorm_backward(e, e, w, torch.empty(0, device=DEV), dw=torch.full((512,), 5.0, device=DEV))
    assert gx.shape == (0, 512) and bool((gw == 0).all())
    assert dx.detox_rmsnorm(e, w, want_q=True).y.shape == (0, 512)
    q, e8 = dx.detox_checkpoint_pack(e)
    assert dx.detox_checkpoint_unpack(q, e8).shape == (0, 512)


# ------------------------------------------------------------------------------------- the gated projections

def act64(name, g):
    if name == "silu":
        s = torch.sigmoid(g)
        return g * s, s * (1 + g * (1 - s))
    if name == "gelu":
        c = 0.5 * torch.erfc(-g / math.sqrt(2))
        return g * c, c + g * torch.exp(-g * g / 2) / math.sqrt(2 * math.pi)
    return g.clamp(min=0), (g > 0).double()


def taken(q, e):
    """What an 8-bit form stands for, in 64 bits."""
    wide = e.float().cpu().double().repeat_interleave(128, 1)[:, : q.shape[1]]
    return q.float().cpu().double() * wide


GATED_SHAPES = [(1, 1, 1), (1, 64, 128), (1, 2048, 300), (2, 8, 130), (5, 100, 77), (48, 256, 512), (127, 72, 129), (128, 64, 128),
                (129, 65, 257), (130, 1000, 33), (300, 513, 391), (1000, 128, 640), (257, 2056, 1031),
                # enough tiles for pairs of CTAs: in the forward pass, for dx, for the weight gradients
                (2100, 72, 1301), (2049, 2401, 41), (33, 2399, 1301)]


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("tokens,in_dim,hidden", GATED_SHAPES)
def test_gated_on_whole_numbers(dtype, tokens, in_dim, hidden):
    """relu and whole numbers: g, u, h and every gradient are exact sums, so only the documented roundings remain."""
    gen = generator(tokens + 3 * in_dim + 5 * hidden)
    keepable = 1.0 if in_dim < 64 else 0.0     # share of non-zero weights small enough that sums stay small
    x = ints(gen, -2, 2, tokens, in_dim)
    wg, wu = (ints(gen, -1, 1, hidden, in_dim) * (torch.rand((hidden, in_dim), generator=gen) < max(keepable, 24.0 / in_dim)) for _ in range(2))
    dh = ints(gen, -2, 2, tokens, hidden)
    for pad, shift in ((0, 0), (3, 1), (8, 8)):
        dev = [strided(t.to(dtype).to(DEV), pad, shift) for t in (x, wg, wu, dh)]
        h, kept = dx.detox_gated(dev[0], dev[1], dev[2], dx.ACT_RELU, keep=True)
        g, u = x @ wg.T, x @ wu.T
        assert torch.equal(h.cpu(), (g.clamp(min=0) * u).to(dtype))
        for v, q, e in ((g, kept.gq, kept.ge), (u, kept.uq, kept.ue)):
            ref_q, ref_e, _ = kept_by_definition(v.numpy())
            assert np.array_equal(e.view(torch.uint8).cpu().numpy(), ref_e)
            assert np.array_equal(q.float().cpu().numpy(), ref_q)
        assert torch.equal(dx.detox_gated(dev[0], dev[1], dev[2], dx.ACT_RELU), h)
        for k in (None, kept):
            G, U = (g, u) if k is None else (taken(kept.gq, kept.ge), taken(kept.uq, kept.ue))
            # dg and du are rounded to the type; their sums are exact while they stay below 2^24
            dg = (dh * U * (G > 0)).to(dtype).double()
            du = (dh * G.clamp(min=0)).to(dtype).double()
            got = dx.detox_gated_backward(dev[3], dev[0], dev[1], dev[2], dx.ACT_RELU, kept=k)
            wide = dx.detox_gated_backward(dev[3], dev[0], dev[1], dev[2], dx.ACT_RELU, kept=k, dw_dtype=F32)
            for name, a, ref in (("dx", got[0], dg @ wg + du @ wu), ("dwg", got[1], dg.T @ x), ("dwu", got[2], du.T @ x)):
                assert torch.equal(a.cpu(), ref.to(dtype)), name
            assert wide[1].dtype == F32 and torch.equal(wide[1].cpu().double(), dg.T @ x) and torch.equal(wide[2].cpu().double(), du.T @ x)


@pytest.mark.parametrize("act", list(ACTS))
@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("tokens,in_dim,hidden", [(1, 2048, 700), (48, 512, 257), (200, 333, 300), (513, 640, 384)])
def test_gated_and_its_gradients(act, dtype, tokens, in_dim, hidden):
    gen = generator(tokens + hidden)
    x = randn(gen, tokens, in_dim).to(dtype)
    wg, wu = (randn(gen, hidden, in_dim, scale=in_dim ** -0.5).to(dtype) for _ in range(2))
    dh = randn(gen, tokens, hidden).to(dtype)
    X, WG, WU, DH = (t.double() for t in (x, wg, wu, dh))
    dev = [t.to(DEV) for t in (x, wg, wu, dh)]
    h, kept = dx.detox_gated(*dev[:3], ACTS[act], keep=True)
    g, u = X @ WG.T, X @ WU.T
    a, da = act64(act, g)
    sums = (in_dim + 8) * 2.0 ** -23
    og, ou = sums * (X.abs() @ WG.abs().T), sums * (X.abs() @ WU.T.abs())
    # act is Lipschitz with 1.2, and computed to 2^-20 of |g|
    oh = (a.abs() + 1.2 * og) * ou + u.abs() * (1.2 * og + 2.0 ** -20 * g.abs())
    unit = HALF_UNIT[dtype]
    within(h, a * u, oh + unit * ((a * u).abs() + oh) + TINY[dtype], "h")
    within(torch.from_numpy(taken(kept.gq, kept.ge).numpy()), g, 2.0 ** -4 * (g.abs() + og) + og + 2.0 ** -10 * kept.ge.float().cpu().double().repeat_interleave(128, 1)[:, :hidden], "kept g")

    for mode in ("again", "kept", "kept, x in 8 bits"):
        xin, k, XB = dev[0], None, X
        if mode != "again":
            k = kept
            G, U = taken(kept.gq, kept.ge), taken(kept.uq, kept.ue)
            eg = eu = torch.zeros_like(G)
        else:
            G, U, eg, eu = g, u, og, ou
        if mode.endswith("8 bits"):
            xin = dx.detox_checkpoint_pack(dev[0])
            XB = taken(*xin)
        A, DA = act64(act, G)
        dg, du = DH * U * DA, DH * A
        # act' is Lipschitz with 1.2 (relu: a step at 0, where |g| is within the error of 0 either value may come out)
        step = (G.abs() <= eg).double() if act == "relu" else 1.2 * eg
        odg = DH.abs() * ((U.abs() + eu) * (step + 2.0 ** -20) + 1.2 * eu) + unit * dg.abs() * 1.01 + TINY[dtype]
        odu = DH.abs() * (1.2 * eg + 2.0 ** -20 * G.abs()) + unit * du.abs() * 1.01 + TINY[dtype]
        got = dx.detox_gated_backward(dev[3], xin, dev[1], dev[2], ACTS[act], kept=k)
        f32 = dx.detox_gated_backward(dev[3], xin, dev[1], dev[2], ACTS[act], kept=k, dw_dtype=F32)
        long = (2 * hidden + 8) * 2.0 ** -23
        size = (dg.abs() + odg) @ WG.abs() + (du.abs() + odu) @ WU.abs()
        ref = dg @ WG + du @ WU
        off = odg @ WG.abs() + odu @ WU.abs() + long * size
        within(got[0], ref, off + unit * (ref.abs() + off) + TINY[dtype], mode + ": dx")
        assert torch.equal(f32[0], got[0])
        for name, i, d, od in (("dwg", 1, dg, odg), ("dwu", 2, du, odu)):
            ref = d.T @ XB
            off = od.T @ XB.abs() + (tokens + 8) * 2.0 ** -23 * ((d.abs() + od).T @ XB.abs())
            within(f32[i], ref, off + 2.0 ** -24 * ref.abs(), mode + ": " + name + " fp32")
            within(got[i], ref, off + unit * (ref.abs() + off) + TINY[dtype], mode + ": " + name)


def test_gated_gradients_against_differences():
    gen = generator(21)
    tokens, in_dim, hidden = 40, 96, 200
    x, wg, wu = randn(gen, tokens, in_dim).to(BF16), randn(gen, hidden, in_dim, scale=0.1).to(BF16), randn(gen, hidden, in_dim, scale=0.1).to(BF16)
    dh = randn(gen, tokens, hidden).to(BF16)
    for act in ("silu", "gelu"):
        got = dx.detox_gated_backward(dh.to(DEV), x.to(DEV), wg.to(DEV), wu.to(DEV), ACTS[act], dw_dtype=F32)

        def loss(x, wg, wu):
            return float((dh.double() * act64(act, x @ wg.T)[0] * (x @ wu.T)).sum())

        at = [x.double(), wg.double(), wu.double()]
        h = 1e-4
        for i in range(3):
            for _ in range(3):
                v = randn(gen, *at[i].shape)
                up, dn = list(at), list(at)
                up[i], dn[i] = at[i] + h * v, at[i] - h * v
                diff = (loss(*up) - loss(*dn)) / (2 * h)
                along = float((got[i].cpu().double() * v).sum())
                # roundings of dg and du (2^-9 each, independent) and of dx; the direction's entries are independent too:
                # six deviations of their sum, and the difference's own error far below that
                assert abs(along - diff) <= 6 * 2.0 ** -8 * float(got[i].cpu().double().norm()), (act, i, along, diff)


def test_weight_gradients_land_in_a_row_of_the_vote_matrix():
    """fp32 weight gradients as pieces of a gradient's row, at an offset that is no multiple of a vector; neighbours stay."""
    gen = generator(31)
    tokens, in_dim, hidden = 70, 96, 130
    x, wg, wu, dh = (randn(gen, *s).to(BF16).to(DEV) for s in ((tokens, in_dim), (hidden, in_dim), (hidden, in_dim), (tokens, hidden)))
    ref = dx.detox_gated_backward(dh, x, wg, wu, dw_dtype=F32)
    n = hidden * in_dim
    for off in (0, 4, 5):
        row = torch.full((2 * n + off + 9,), 7.0, device=DEV)
        a, b = row[off: off + n].view(hidden, in_dim), row[off + n: off + 2 * n].view(hidden, in_dim)
        dx.detox_gated_backward(dh, x, wg, wu, dwg=a, dwu=b)
        assert torch.equal(a, ref[1]) and torch.equal(b, ref[2])
        assert bool((row[:off] == 7.0).all()) and bool((row[off + 2 * n:] == 7.0).all())


def test_gated_outputs_leave_padding_alone_and_zero_tokens_work():
    gen = generator(32)
    x, wg, wu, dh = (randn(gen, *s).to(F16).to(DEV) for s in ((131, 72), (140, 72), (140, 72), (131, 140)))
    h = dx.detox_gated(x, wg, wu)
    for pad in (1, 8):
        buf = torch.full((131, 140 + pad), 7.0, dtype=F16, device=DEV)
        dx.detox_gated(x, wg, wu, h=buf[:, :140])
        assert torch.equal(buf[:, :140], h) and bool((buf[:, 140:] == 7.0).all())
        gx = torch.full((131, 72 + pad), 7.0, dtype=F16, device=DEV)
        gw = [torch.full((140, 72 + pad), 7.0, dtype=F16, device=DEV) for _ in range(2)]
        dx.detox_gated_backward(dh, x, wg, wu, dx=gx[:, :72], dwg=gw[0][:, :72], dwu=gw[1][:, :72])
        for t in (gx, *gw):
            assert bool((t[:, 72:] == 7.0).all()) and not bool((t[:, :72] == 7.0).all())
        e = x[:0]
        assert dx.detox_gated(e, wg, wu).shape == (0, 140)
        g0, a, b = dx.detox_gated_backward(dh[:0], e, wg, wu, dwg=gw[0][:, :72], dwu=gw[1][:, :72])
        assert g0.shape == (0, 72) and bool((a == 0).all()) and bool((b == 0).all())
        assert all(bool((t[:, 72:] == 7.0).all()) for t in gw)


def test_tokens_do_not_meet():
    """A token of NaN or Inf changes no other token's h or dx."""
    gen = generator(33)
    x, wg, wu, dh = (randn(gen, *s).to(BF16).to(DEV) for s in ((200, 128), (256, 128), (256, 128), (200, 256)))
    h, gx = dx.detox_gated(x, wg, wu), dx.detox_gated_backward(dh, x, wg, wu)[0]
    bad = x.clone()
    bad[5] = math.nan
    bad[150, 3] = math.inf
    h2, gx2 = dx.detox_gated(bad, wg, wu), dx.detox_gated_backward(dh, bad, wg, wu)[0]
    rest = [i for i in range(200) if i not in (5, 150)]
    assert torch.equal(h2[rest], h[rest]) and torch.equal(gx2[rest], gx[rest])
    assert bool(h2[5].isnan().all())


def test_same_bits_every_time_on_another_stream_and_in_a_graph():
    gen = generator(34)
    x, wg, wu, dh = (randn(gen, *s).to(BF16).to(DEV) for s in ((700, 320), (520, 320), (520, 320), (700, 520)))
    w = randn(gen, 320).to(BF16).to(DEV)

    def step():
        n = dx.detox_rmsnorm(x, w, want_q=True)
        h, kept = dx.detox_gated(n.y, wg, wu, keep=True)
        gy, a, b = dx.detox_gated_backward(dh, (n.q, n.e), wg, wu, kept=kept, dw_dtype=F32)
        gx, gw = dx.detox_rmsnorm_backward(gy, x, w, n.rstd)
        return [n.y, h, gy, a, b, gx, gw]

    first = step()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        again = step()
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(first, again))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step()
    for t in out:
        t.zero_()
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(first, out))


def test_status_word_reads_zero():
    gen = generator(35)
    x, wg, wu, dh = (randn(gen, *s).to(BF16).to(DEV) for s in ((300, 64), (200, 64), (200, 64), (300, 200)))
    ws = torch.full((dx.detox_gated_workspace_bytes(x, wg, wu),), 0x5A, dtype=torch.uint8, device=DEV)
    dx.detox_gated(x, wg, wu, ws=ws)
    assert dx.read_status(ws) == 0
    ws = torch.full((dx.detox_gated_backward_workspace_bytes(x, wg, wu),), 0x5A, dtype=torch.uint8, device=DEV)
    dx.detox_gated_backward(dh, x, wg, wu, ws=ws)
    assert dx.read_status(ws) == 0
    dx.check_status(ws)


def test_inf_and_nan_in_kept_projections():
    """Inf and NaN among g and u are kept as NaN, and a block's scale comes from its finite entries: in the epilogue of a tile
    of its own and in that of a tile whose reduction is split."""
    gen = generator(41)
    for tokens, in_dim in ((300, 64), (3, 1024), (2100, 64)):
        x, wg, wu = ints(gen, -2, 2, tokens, in_dim), ints(gen, -1, 1, 700, in_dim), ints(gen, -1, 1, 700, in_dim)
        wg[5, :] = math.inf       # g[:, 5] = +-Inf or NaN
        wu[300, 0] = math.nan
        dev = [t.to(BF16).to(DEV) for t in (x, wg, wu)]
        _, kept = dx.detox_gated(*dev, dx.ACT_RELU, keep=True)
        for w, q, e, bad in ((wg, kept.gq, kept.ge, 5), (wu, kept.uq, kept.ue, 300)):
            fine = w.clone()
            fine[bad] = 0.0
            v = x @ fine.T
            ref_q, ref_e, _ = kept_by_definition(v.numpy())
            got = q.float().cpu().numpy()
            assert np.isnan(got[:, bad]).all()
            got[:, bad] = ref_q[:, bad] = 0.0
            assert np.array_equal(got, ref_q) and np.array_equal(e.view(torch.uint8).cpu().numpy(), ref_e)


@pytest.mark.parametrize("tokens,in_dim,hidden", [(9, 600, 300), (300, 100, 260), (2050, 64, 1400)])
def test_kept_buffers_of_any_alignment(tokens, in_dim, hidden):
    """Kept buffers with odd strides and offsets, which the C interface allows, hold and give back the same."""
    import ctypes
    gen = generator(42)
    x, wg, wu, dh = (randn(gen, *s).to(F16).to(DEV) for s in ((tokens, in_dim), (hidden, in_dim), (hidden, in_dim), (tokens, hidden)))
    h, kept = dx.detox_gated(x, wg, wu, dx.ACT_GELU, keep=True)
    nb = -(-hidden // 128)
    ldq, lde = hidden + 3, nb + 1
    q = torch.full((2 * tokens * ldq + 8,), 9, dtype=torch.uint8, device=DEV)
    e = torch.full((2 * tokens * lde + 8,), 9, dtype=torch.uint8, device=DEV)
    vq = [q[1 + i * tokens * ldq: 1 + (i + 1) * tokens * ldq].view(tokens, ldq) for i in range(2)]
    ve = [e[i * tokens * lde: (i + 1) * tokens * lde].view(tokens, lde) for i in range(2)]
    d = dx.GatedDesc(dx.DTYPE_HALF, dx.ACT_GELU, tokens, in_dim, hidden, x.data_ptr(), x.stride(0), None, 0, None, 0, wg.data_ptr(), wg.stride(0),
                     wu.data_ptr(), wu.stride(0), vq[0].data_ptr(), ve[0].data_ptr(), vq[1].data_ptr(), ve[1].data_ptr(), ldq, lde)
    lib = dx.load()
    ws = torch.empty(max(lib.detox_gated_workspace_bytes(ctypes.byref(d)), 256), dtype=torch.uint8, device=DEV)
    h2 = torch.empty_like(h)
    assert lib.detox_gated(ctypes.byref(d), h2.data_ptr(), h2.stride(0), ws.data_ptr(), ws.numel(), torch.cuda.current_stream().cuda_stream) == 0
    assert torch.equal(h2, h)
    for i, (a, b) in enumerate(((kept.gq, kept.ge), (kept.uq, kept.ue))):
        assert torch.equal(vq[i][:, :hidden], a.view(torch.uint8)) and torch.equal(ve[i][:, :nb], b.view(torch.uint8))
        assert bool((vq[i][:, hidden:] == 9).all()) and bool((ve[i][:, nb:] == 9).all())
    f8, e8 = q[1: 1 + 2 * tokens * ldq].view(torch.float8_e4m3fn).view(2, tokens, ldq), e[: 2 * tokens * lde].view(torch.float8_e8m0fnu).view(2, tokens, lde)
    odd = dx.Kept(f8[:, :, :hidden], e8[:, :, :nb])
    for a, b in zip(dx.detox_gated_backward(dh, x, wg, wu, dx.ACT_GELU, kept=kept), dx.detox_gated_backward(dh, x, wg, wu, dx.ACT_GELU, kept=odd)):
        assert torch.equal(a, b)


def test_calls_one_after_another_on_the_same_buffers():
    """Kernels start while the ones before them finish; calls that reuse outputs and workspace must not meet."""
    gen = generator(43)
    shapes = ((260, 512), (1408, 512), (1408, 512), (260, 1408))
    sets = [[randn(gen, *s).to(BF16).to(DEV) for s in shapes] for _ in range(3)]
    want = []
    for x, wg, wu, dh in sets:
        want.append([t.clone() for t in dx.detox_gated_backward(dh, x, wg, wu)])
        torch.cuda.synchronize()
    outs = [torch.empty_like(t) for t in want[0]]
    ws = torch.empty(dx.detox_gated_backward_workspace_bytes(*sets[0][:3]), dtype=torch.uint8, device=DEV)
    copies = []
    for k in range(30):
        x, wg, wu, dh = sets[k % 3]
        dx.detox_gated_backward(dh, x, wg, wu, dx=outs[0], dwg=outs[1], dwu=outs[2], ws=ws)
        if k >= 24:
            copies.append((k % 3, [t.clone() for t in outs]))
    # a chain in which each call reads what the one before it wrote
    y = dx.detox_rmsnorm(sets[0][0], sets[0][1][0].contiguous()).y
    for _ in range(10):
        y = dx.detox_rmsnorm(y, sets[0][1][0].contiguous(), residual=sets[0][0]).y
        q, e = dx.detox_checkpoint_pack(y)
        y = dx.detox_checkpoint_unpack(q, e, BF16)
    torch.cuda.synchronize()
    for which, got in copies:
        assert all(torch.equal(a, b) for a, b in zip(got, want[which]))
    z = dx.detox_rmsnorm(sets[0][0], sets[0][1][0].contiguous()).y
    for _ in range(10):
        torch.cuda.synchronize()
        z = dx.detox_rmsnorm(z, sets[0][1][0].contiguous(), residual=sets[0][0]).y
        torch.cuda.synchronize()
        q, e = dx.detox_checkpoint_pack(z)
        torch.cuda.synchronize()
        z = dx.detox_checkpoint_unpack(q, e, BF16)
    assert torch.equal(y, z)


def test_offsets_that_pass_32_bits():
    """More than 2^32 entries of h: the first and last tokens are the ones of a small call, and so are their gradients."""
    tokens, in_dim, hidden = 1_050_000, 64, 4096 + 8
    g = torch.Generator(device=DEV).manual_seed(7)
    x = torch.randn((tokens, in_dim), generator=g, device=DEV, dtype=torch.float32).to(BF16)
    wg, wu = (torch.randn((hidden, in_dim), generator=g, device=DEV).mul_(0.125).to(BF16) for _ in range(2))
    h = dx.detox_gated(x, wg, wu)
    ends = torch.cat([torch.arange(300, device=DEV), torch.arange(tokens - 300, tokens, device=DEV)])
    few = x[ends].contiguous()
    ref = (torch.nn.functional.silu(few.double() @ wg.double().T) * (few.double() @ wu.double().T))
    # silu is Lipschitz with 1.1; sums of 64 products of size up to 20
    assert bool(((h[ends].double() - ref).abs() <= 2.0 ** -8 * ref.abs() + 1e-3).all())
    dh = h
    gx, a, b = dx.detox_gated_backward(dh, x, wg, wu, dw_dtype=F32)
    few_gx = dx.detox_gated_backward(dh[ends].contiguous(), few, wg, wu)[0]
    assert bool(((gx[ends].double() - few_gx.double()).norm(dim=1) <= 2.0 ** -7 * few_gx.double().norm(dim=1)).all())
    # dWu over all tokens, for the last rows of the weight: du = dh act(g), rounded to bf16
    last = slice(hidden - 3, hidden)
    total = torch.zeros((3, in_dim), dtype=torch.float64, device=DEV)
    size = torch.zeros((3, in_dim), dtype=torch.float64, device=DEV)
    for k in range(0, tokens, 150_000):
        xs, ds = x[k: k + 150_000].double(), dh[k: k + 150_000, last].double()
        du = ds * torch.nn.functional.silu(xs @ wg[last].double().T)
        total += du.T @ xs
        size += du.abs().T @ xs.abs()
    # a rounding of 2^-8 in each du, and an fp32 chain over the tokens
    assert bool(((b[last].double() - total).abs() <= (2.0 ** -8 + tokens * 2.0 ** -23) * size).all())
    del h, dh, gx

    rows = 1_100_000
    x = torch.randn((rows, 4096), generator=g, device=DEV, dtype=F16)
    w = torch.ones(4096, device=DEV, dtype=F16)
    got = dx.detox_rmsnorm(x, w, want_y=True)
    few = dx.detox_rmsnorm(x[-5:].contiguous(), w)
    assert torch.equal(got.y[-5:], few.y) and torch.equal(got.rstd[-5:], few.rstd)


@pytest.mark.parametrize("act", list(ACTS))
@pytest.mark.parametrize("tokens", [3, 300])
def test_nan_reaches_its_own_outputs(act, tokens):
    """A NaN in a token makes that token's h, dx and all weight gradients NaN, whatever the activation; a NaN in dh does so for its
    row of the weight gradients and its token's dx."""
    gen = generator(51)
    x, wg, wu, dh = (randn(gen, *s).to(BF16).to(DEV) for s in ((tokens, 96), (140, 96), (140, 96), (tokens, 140)))
    bad = x.clone()
    bad[1, 7] = math.nan
    h, kept = dx.detox_gated(bad, wg, wu, ACTS[act], keep=True)
    assert bool(h[1].isnan().all()) and not bool(h[0].isnan().any())
    for k in (None, kept):
        gx, a, b = dx.detox_gated_backward(dh, bad, wg, wu, ACTS[act], kept=k)
        assert bool(gx[1].isnan().all()) and not bool(gx[0].isnan().any()) and bool(b.isnan().all())
    hurt = dh.clone()
    hurt[1, 5] = math.nan
    gx, a, b = dx.detox_gated_backward(hurt, x, wg, wu, ACTS[act])
    assert bool(gx[1].isnan().all()) and not bool(gx[0].isnan().any())
    assert bool(b[5].isnan().all()) and not bool(b[4].isnan().any()) and not bool(b[6].isnan().any())


@pytest.mark.parametrize("tokens,in_dim,hidden", [(1, 64, 128), (70, 97, 131), (520, 512, 300), (2100, 64, 1300)])
def test_workspaces_are_as_large_as_they_say(tokens, in_dim, hidden):
    """With exactly the bytes the helpers ask for, between guard bands that nothing may touch."""
    gen = generator(52)
    x, wg, wu, dh = (randn(gen, *s).to(F16).to(DEV) for s in ((tokens, in_dim), (hidden, in_dim), (hidden, in_dim), (tokens, hidden)))

    def guarded(n):
        buf = torch.full((n + 8192,), 0xA5, dtype=torch.uint8, device=DEV)
        return buf, buf[4096: 4096 + n]

    def intact(buf, n):
        return bool((buf[:4096] == 0xA5).all()) and bool((buf[4096 + n:] == 0xA5).all())

    pair = dx.detox_checkpoint_pack(x)
    for xin in (x, pair):
        n = dx.detox_gated_workspace_bytes(xin, wg, wu)
        buf, ws = guarded(n)
        h, kept = dx.detox_gated(xin, wg, wu, keep=True, ws=ws)
        assert intact(buf, n)
        for k in (None, kept):
            n = dx.detox_gated_backward_workspace_bytes(xin, wg, wu, kept=k)
            buf, ws = guarded(n)
            dx.detox_gated_backward(dh, xin, wg, wu, kept=k, ws=ws)
            assert intact(buf, n)
    for dtype in (F16, F32):
        n = dx.detox_rmsnorm_backward_workspace_bytes(tokens, in_dim)
        buf, ws = guarded(n)
        dx.detox_rmsnorm_backward(x.to(dtype), x.to(dtype), wg[0].to(dtype).contiguous(), torch.ones(tokens, device=DEV), ws=ws)
        assert intact(buf, n)
    with pytest.raises(dx.DetoxError) as e:
        dx.detox_gated(x, wg, wu, ws=torch.empty(0, dtype=torch.uint8, device=DEV))
    assert e.value.code == 3


def test_refusals_of_the_binding():
    x, w = torch.zeros((8, 64), dtype=BF16, device=DEV), torch.zeros((32, 64), dtype=BF16, device=DEV)
    dh = torch.zeros((8, 32), dtype=BF16, device=DEV)
    for wrong in (lambda: dx.detox_gated(x.float(), w, w), lambda: dx.detox_gated(x, w, w.half()), lambda: dx.detox_gated(x[0], w, w),
                  lambda: dx.detox_rmsnorm(x, w), lambda: dx.detox_rmsnorm(x.int(), w[0]), lambda: dx.detox_checkpoint_pack(x.double()),
                  lambda: dx.detox_checkpoint_unpack(x, x), lambda: dx.detox_gated_backward(dh, x, w, w, dw_dtype=torch.int32),
                  lambda: dx.detox_rmsnorm_backward(x, x, w[0], torch.zeros(7, device=DEV)), lambda: dx.detox_gated(None, w, w)):
        with pytest.raises(TypeError):
            wrong()
    for wrong in (lambda: dx.detox_gated(x[:, :32], w, w), lambda: dx.detox_gated(x.T, x.T, x.T), lambda: dx.detox_gated(x, w, w[:8]),
                  lambda: dx.detox_gated_backward(dh[:4], x, w, w), lambda: dx.detox_gated_backward(dh, x, w, w, dwg=torch.zeros_like(w)),
                  lambda: dx.detox_rmsnorm(x, w[0].contiguous(), residual=x[:4]), lambda: dx.detox_rmsnorm(x, w[0].contiguous(), sum_out=x)):
        with pytest.raises(ValueError):
            wrong()
    with pytest.raises(dx.DetoxError) as e:
        dx.detox_gated(x.float(), w.float(), w.float())
    assert e.value.code == 2                       # the tensor cores multiply 16-bit entries
    with pytest.raises(dx.DetoxError) as e:
        dx.detox_gated(x, w, w, act=9)
    assert e.value.code == 1
    with pytest.raises(dx.DetoxError) as e:
        wide = torch.zeros((2, 40000), dtype=BF16, device=DEV)
        dx.detox_rmsnorm(wide, wide[0].contiguous())
    assert e.value.code == 2
