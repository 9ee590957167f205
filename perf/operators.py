"""What is measured of the worker-side operators: a worker's gated feed-forward sublayer and the 8-bit checkpoints of its
activations.

A DETOX worker computes the gradient that the parameter server votes on.  The operators here are the ones of a pre-norm
feed-forward sublayer: the root-mean-square norm with the residual's addition, the gated pair of projections, and the
8-bit form in which activations are kept between the forward and the backward pass.

`run` computes each case in its plain form (torch, 32 bits, rounded once at the end) or, where `own` is true, through the
framework's entry points.  Matrices have rows of tokens; weights are [out, in], as a linear layer keeps them.
"""
import math

import torch

own = False

_DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
_BLOCK = 128          # columns that share a scale
_E4M3_MAX = 448.0
_EPS = 1e-6


# ---------------------------------------------------------------------------------------------- cases

def listed():
    return [
        # one token of a decoder whose next product takes 8-bit rows: the call's latency is what counts
        {"name": "norm_token", "op": "norm", "dtype": "bf16", "rows": 1, "cols": 2048, "pad": 0, "residual": True, "y": True, "q": True},
        # a training batch; the normed rows leave in 8 bits only, as the checkpoint of the products that follow
        {"name": "norm_batch", "op": "norm", "dtype": "bf16", "rows": 8192, "cols": 4096, "pad": 0, "residual": True, "y": False, "q": True},
        # a ragged batch of rows cut out of a wider fp16 buffer, width no multiple of the 8-bit block nor of a vector load
        {"name": "norm_odd", "op": "norm", "dtype": "f16", "rows": 1023, "cols": 1111, "pad": 9, "residual": False, "y": True, "q": False},
        # its backward pass over a training batch, with the residual stream's own gradient added in
        {"name": "norm_grad", "op": "norm_grad", "dtype": "bf16", "rows": 8192, "cols": 2048, "pad": 0, "residual": True},
        # the hidden activations of a batch laid away in 8 bits
        {"name": "keep_batch", "op": "keep", "dtype": "bf16", "rows": 8192, "cols": 5632, "pad": 0, "back": False},
        # rows of an odd pitch kept and taken out again
        {"name": "keep_odd", "op": "keep", "dtype": "f16", "rows": 777, "cols": 1003, "pad": 3, "back": True},
        # one token through both projections: bound by reading the weights
        {"name": "gated_token", "op": "gated", "dtype": "bf16", "act": "silu", "rows": 1, "cols": 2048, "hidden": 5632, "pad": 0},
        # a few dozen sequences decoded together
        {"name": "gated_few", "op": "gated", "dtype": "f16", "act": "gelu", "rows": 48, "cols": 1024, "hidden": 2816, "pad": 0},
        # a prompt, or a validation batch
        {"name": "gated_prompt", "op": "gated", "dtype": "bf16", "act": "silu", "rows": 4096, "cols": 2048, "hidden": 5632, "pad": 0},
        # a small worker's step: forward, activations kept in 8 bits, backward from them
        {"name": "step_small", "op": "step", "dtype": "bf16", "act": "gelu", "rows": 500, "cols": 512, "hidden": 1408, "pad": 0, "kept": True},
        # backward without kept activations (both projections computed again), sizes no multiple of any tile or vector
        {"name": "step_odd", "op": "step", "dtype": "f16", "act": "silu", "rows": 1001, "cols": 1000, "hidden": 2730, "pad": 4, "kept": False},
        # the step of a full batch
        {"name": "step_batch", "op": "step", "dtype": "bf16", "act": "silu", "rows": 8192, "cols": 2048, "hidden": 5632, "pad": 0, "kept": True},
    ]


def draw(rng):
    def size(lo, hi):
        """Spread over the logarithm; a third of them odd, a third round."""
        v = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
        kind = rng.randrange(3)
        if kind == 0:
            v |= 1
        elif kind == 1 and v >= 64:
            v = v // 64 * 64
        return max(lo, min(hi, v))

    op = rng.choice(["norm", "norm", "norm_grad", "keep", "gated", "gated", "step", "step"])
    case = {"op": op, "dtype": rng.choice(["bf16", "f16"]), "pad": rng.choice([0, 0, 1, 5, 8])}
    if op in ("norm", "norm_grad", "keep"):
        case["dtype"] = rng.choice(["bf16", "f16", "f32"])
        case["rows"], case["cols"] = size(1, 8192), size(64, 4096)
        if op == "norm":
            q = rng.random() < 0.6
            case |= {"residual": rng.random() < 0.6, "q": q, "y": not q or rng.random() < 0.5}
        elif op == "norm_grad":
            case["residual"] = rng.random() < 0.6
        else:
            case["back"] = rng.random() < 0.5
        return case
    case |= {"act": rng.choice(["silu", "gelu", "relu"]), "rows": size(1, 8192), "cols": size(64, 2048), "hidden": size(64, 5632)}
    if op == "step":
        case["kept"] = rng.random() < 0.5
    return case


def work(case):
    """The least a pass has to read, write and compute.  The 8-bit form of a row takes a byte an entry and one for each block's scale."""
    size = 4 if case["dtype"] == "f32" else 2
    t, k = case["rows"], case["cols"]
    eight = t * k + t * -(-k // _BLOCK)
    if case["op"] == "norm":
        moved = t * k * size * (1 + 2 * case["residual"] + case["y"]) + k * size + 4 * t + eight * case["q"]
        return {"bytes": moved, "flops": 6 * t * k}
    if case["op"] == "norm_grad":
        return {"bytes": t * k * size * (3 + case["residual"]) + k * (size + 4) + 4 * t, "flops": 10 * t * k}
    if case["op"] == "keep":
        return {"bytes": t * k * size * (1 + case["back"]) + eight, "flops": 3 * t * k}
    f = case["hidden"]
    if case["op"] == "gated":
        return {"bytes": size * (t * k + 2 * f * k + t * f), "flops": 4 * t * k * f}
    # x, both weights and dh read; h (of a forward pass), dx and both weight gradients written
    moved = size * (2 * t * k + 4 * f * k + t * f * (1 + case["kept"]))
    return {"bytes": moved, "flops": 12 * t * k * f}


# ---------------------------------------------------------------------------------------------- inputs

def _matrix(gen, rows, cols, pad, dtype, scale=1.0):
    """A matrix whose rows lie cols + pad entries apart."""
    m = torch.randn((rows, cols + pad), generator=gen, device="cuda", dtype=torch.float32)
    return m.mul_(scale).to(dtype)[:, :cols]


def _activations(gen, rows, cols, pad, dtype):
    """Rows as a residual stream has them: tokens of different size, and a few channels that stand out."""
    m = torch.randn((rows, cols + pad), generator=gen, device="cuda", dtype=torch.float32)
    m *= torch.exp(0.5 * torch.randn((rows, 1), generator=gen, device="cuda"))
    loud = torch.rand((1, cols + pad), generator=gen, device="cuda") < 0.01
    return torch.where(loud, 12.0 * m, m).to(dtype)[:, :cols]


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(int(seed))
    dtype, t, k, pad = _DTYPES[case["dtype"]], case["rows"], case["cols"], case["pad"]
    s = {"case": dict(case)}
    if case["op"] == "keep":
        s["x"] = _activations(gen, t, k, pad, dtype)
        return s
    if case["op"] in ("norm", "norm_grad"):
        s["x"] = _activations(gen, t, k, pad, dtype)
        s["w"] = (1.0 + 0.2 * torch.randn(k, generator=gen, device="cuda")).to(dtype)
        if case["op"] == "norm":
            s["residual"] = _activations(gen, t, k, pad, dtype) if case["residual"] else None
        else:
            # what the forward pass left: the sum (here x itself) and 1 / its root mean square
            x = s["x"].float()
            s["rstd"] = torch.rsqrt((x * x).mean(1) + _EPS)
            s["dy"] = _matrix(gen, t, k, pad, dtype)
            s["ds"] = _matrix(gen, t, k, pad, dtype) if case["residual"] else None
        return s
    f = case["hidden"]
    x = torch.randn((t, k + pad), generator=gen, device="cuda")
    s["x"] = x.to(dtype)[:, :k]                                    # normed rows
    s["wg"] = _matrix(gen, f, k, 0, dtype, 1.0 / math.sqrt(k))
    s["wu"] = _matrix(gen, f, k, 0, dtype, 1.0 / math.sqrt(k))
    if case["op"] == "step":
        s["dh"] = _matrix(gen, t, f, pad, dtype)
    return s


# ---------------------------------------------------------------------------------------------- plain forms

def _scales(x):
    """Exponents e of the power-of-two scales: the smallest with amax <= 448 * 2^e in each block of 128 columns."""
    t, k = x.shape
    n = -(-k // _BLOCK)
    a = torch.nn.functional.pad(x.abs(), (0, n * _BLOCK - k)).reshape(t, n, _BLOCK)
    m, e = torch.frexp(a.amax(2))                                  # amax = m 2^e, 0.5 <= m < 1
    return torch.where(m <= 0.875, e - 9, e - 8).clamp(min=-126)


def _kept(x):
    """8-bit form of fp32 rows: (values, scales)."""
    e = _scales(x)
    wide = e.repeat_interleave(_BLOCK, 1)[:, : x.shape[1]]
    q = torch.ldexp(x, -wide).to(torch.float8_e4m3fn)
    return q, torch.ldexp(torch.ones_like(e, dtype=torch.float32), e).to(torch.float8_e8m0fnu)


def _taken(q, e):
    return q.float() * e.float().repeat_interleave(_BLOCK, 1)[:, : q.shape[1]]


def _act(name, g):
    """The activation and its derivative."""
    if name == "silu":
        s = 1.0 / (1.0 + torch.exp(-g))
        return g * s, s * (1.0 + g * (1.0 - s))
    if name == "gelu":
        c = 0.5 * (1.0 + torch.erf(g * math.sqrt(0.5)))
        return g * c, c + g * torch.exp(-0.5 * g * g) * (1.0 / math.sqrt(2.0 * math.pi))
    r = (g > 0).to(g.dtype)
    return g * r, r


def _plain(s):
    c = s["case"]
    dtype = _DTYPES[c["dtype"]]
    x = s["x"].float()
    if c["op"] == "norm":
        if s["residual"] is not None:
            x = x + s["residual"].float()
        rstd = torch.rsqrt((x * x).mean(1) + _EPS)
        y = x * rstd[:, None] * s["w"].float()
        out = {"rstd": rstd}
        if s["residual"] is not None:
            out["sum"] = x.to(dtype)
        if c["y"]:
            out["y"] = y.to(dtype)
        if c["q"]:
            out["q"], out["e"] = _kept(y)
        return out
    if c["op"] == "norm_grad":
        dy, rstd = s["dy"].float(), s["rstd"][:, None]
        hat = x * rstd
        dyw = dy * s["w"].float()
        dx = rstd * (dyw - hat * (dyw * hat).mean(1, keepdim=True))
        if s["ds"] is not None:
            dx = dx + s["ds"].float()
        return {"dx": dx.to(dtype), "dw": (dy * hat).sum(0)}
    if c["op"] == "keep":
        q, e = _kept(x)
        out = {"q": q, "e": e}
        if c["back"]:
            out["x"] = _taken(q, e).to(dtype)
        return out
    wg, wu = s["wg"].float(), s["wu"].float()
    g, u = x @ wg.T, x @ wu.T
    a, da = _act(c["act"], g)
    h = (a * u).to(dtype)
    if c["op"] == "gated":
        return {"h": h}
    out = {}
    if c["kept"]:
        out["h"] = h
        x, g, u = _taken(*_kept(x)), _taken(*_kept(g)), _taken(*_kept(u))
        a, da = _act(c["act"], g)
    dh = s["dh"].float()
    dg, du = dh * u * da, dh * a
    out |= {"dx": (dg @ wg + du @ wu).to(dtype), "dwg": (dg.T @ x).to(dtype), "dwu": (du.T @ x).to(dtype)}
    return out


# ---------------------------------------------------------------------------------------------- the framework's calls

def _own(s):
    import paper_1907_12205_b200 as dx
    c = s["case"]
    if c["op"] == "norm":
        r = dx.detox_rmsnorm(s["x"], s["w"], residual=s["residual"], eps=_EPS, want_y=c["y"], want_q=c["q"])
        out = {"rstd": r.rstd}
        if s["residual"] is not None:
            out["sum"] = r.sum
        if c["y"]:
            out["y"] = r.y
        if c["q"]:
            out["q"], out["e"] = r.q, r.e
        return out
    if c["op"] == "norm_grad":
        gx, gw = dx.detox_rmsnorm_backward(s["dy"], s["x"], s["w"], s["rstd"], ds=s["ds"])
        return {"dx": gx, "dw": gw}
    if c["op"] == "keep":
        q, e = dx.detox_checkpoint_pack(s["x"])
        out = {"q": q, "e": e}
        if c["back"]:
            out["x"] = dx.detox_checkpoint_unpack(q, e, s["x"].dtype)
        return out
    act = {"silu": dx.ACT_SILU, "gelu": dx.ACT_GELU, "relu": dx.ACT_RELU}[c["act"]]
    if c["op"] == "gated":
        return {"h": dx.detox_gated(s["x"], s["wg"], s["wu"], act)}
    out, x, kept = {}, s["x"], None
    if c["kept"]:
        out["h"], kept = dx.detox_gated(x, s["wg"], s["wu"], act, keep=True)
        x = dx.detox_checkpoint_pack(x)
    out["dx"], out["dwg"], out["dwu"] = dx.detox_gated_backward(s["dh"], x, s["wg"], s["wu"], act, kept=kept)
    return out


def run(state):
    return _own(state) if own else _plain(state)


# ---------------------------------------------------------------------------------------------- 64 bits

def exact(case, seed):
    """The definitions in 64 bits, on the inputs of this seed."""
    s = prepare(case, seed)
    x = s["x"].double()

    def eight(v):
        """What the 8-bit form of v stands for, as (values, scales): four significant bits, steps of 2^-9 below 2^-6."""
        t, k = v.shape
        n = (k + _BLOCK - 1) // _BLOCK
        scale = torch.empty((t, n), dtype=torch.float64, device=v.device)
        q = torch.empty_like(v)
        for b in range(n):
            part = v[:, b * _BLOCK:(b + 1) * _BLOCK]
            amax = part.abs().max(1).values
            e = torch.ceil(torch.log2(torch.clamp(amax, min=1e-300) / _E4M3_MAX))
            e = torch.where(amax > _E4M3_MAX * torch.exp2(e), e + 1, e)
            e = torch.where(amax <= _E4M3_MAX * torch.exp2(e - 1), e - 1, e).clamp(min=-126)
            scale[:, b] = torch.exp2(e)
            p = part / torch.exp2(e)[:, None]
            step = torch.exp2(torch.floor(torch.log2(torch.clamp(p.abs(), min=2.0 ** -6))) - 3)
            q[:, b * _BLOCK:(b + 1) * _BLOCK] = torch.round(p / step) * step
        return q, scale

    def back(q, scale):
        return q * scale.repeat_interleave(_BLOCK, dim=1)[:, : q.shape[1]]

    op = case["op"]
    if op == "keep":
        q, e = eight(x)
        return {"q": q, "e": e, "x": back(q, e)} if case["back"] else {"q": q, "e": e}
    if op == "norm":
        if case["residual"]:
            x = x + s["residual"].double()
        rms = torch.sqrt((x ** 2).sum(1) / x.shape[1] + _EPS)
        y = x / rms[:, None] * s["w"].double()
        out = {"rstd": 1.0 / rms}
        if case["residual"]:
            out["sum"] = x
        if case["y"]:
            out["y"] = y
        if case["q"]:
            out["q"], out["e"] = eight(y)
        return out
    if op == "norm_grad":
        dy, r, w = s["dy"].double(), s["rstd"].double()[:, None], s["w"].double()
        inner = (dy * w * x).sum(1, keepdim=True)
        dx = r * w * dy - (r ** 3) * x * inner / x.shape[1]
        if case["residual"]:
            dx = dx + s["ds"].double()
        return {"dx": dx, "dw": torch.einsum("tk,tk,t->k", dy, x, r[:, 0])}
    wg, wu = s["wg"].double(), s["wu"].double()

    def act(g):
        if case["act"] == "silu":
            sg = torch.sigmoid(g)
            return g * sg, sg + g * sg * (1.0 - sg)
        if case["act"] == "gelu":
            cdf = 0.5 * torch.erfc(-g / math.sqrt(2.0))
            return g * cdf, cdf + g * torch.exp(-g * g / 2.0) / math.sqrt(2.0 * math.pi)
        return torch.clamp(g, min=0.0), torch.where(g > 0, 1.0, 0.0).double()

    g, u = torch.matmul(x, wg.t()), torch.matmul(x, wu.t())
    out = {}
    if op == "gated" or case["kept"]:
        out["h"] = act(g)[0] * u
    if op == "gated":
        return out
    if case["kept"]:
        x, g, u = back(*eight(x)), back(*eight(g)), back(*eight(u))
    a, da = act(g)
    dh = s["dh"].double()
    dg, du = dh * u * da, dh * a
    out["dx"] = torch.matmul(dg, wg) + torch.matmul(du, wu)
    out["dwg"], out["dwu"] = torch.matmul(dg.t(), x), torch.matmul(du.t(), x)
    return out
