"""What is measured of the operators around a worker's sublayer: the token embedding, the losses over logits, and the optimizer's
step that takes an aggregated gradient into the weights.

  embedding    rows of a table, scaled; its gradient adds the rows of equal tokens in a fixed order
  logp         log-probabilities of chosen tokens, and their gradient
  policy       the clipped policy loss with a KL term, with the gradient of the logits
  preference   the loss of paired log ratios over packed sequences, with the gradient of the logits
  adamw        one step over many tensors, slices of flat vectors, with states in 32 bits or in 8

`run` computes each case in its plain form (torch, 32 bits or 64, rounded once at the end) or, where `own` is true, through the
framework's entry points.
"""
import math

import torch

own = False

_DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
_BLOCK = 128          # entries of an 8-bit state that share a scale
_BETA1, _BETA2, _EPS = 0.9, 0.999, 1e-8
_CLIP_LOW, _CLIP_HIGH, _KL = 0.2, 0.28, 0.05
_PAIR_BETA, _SMOOTH = 0.1, 0.05


# ---------------------------------------------------------------------------------------------- cases

def listed():
    return [
        # the next token of one sequence: the call's latency is what counts
        {"name": "embed_token", "op": "embed", "dtype": "bf16", "tokens": 1, "vocab": 32000, "cols": 2048, "pad": 0},
        # a training batch
        {"name": "embed_batch", "op": "embed", "dtype": "bf16", "tokens": 8192, "vocab": 32000, "cols": 4096, "pad": 0},
        # the table's gradient of a batch, fp32, as a piece of the row that is sent to the vote
        {"name": "embed_grad_batch", "op": "embed_grad", "dtype": "bf16", "tokens": 8192, "vocab": 32000, "cols": 2048, "pad": 0,
         "wide": True, "add": False},
        # a ragged batch added to the gradient of a tied output head, widths no multiple of a vector load
        {"name": "embed_grad_tied", "op": "embed_grad", "dtype": "f16", "tokens": 1501, "vocab": 5003, "cols": 1003, "pad": 2,
         "wide": False, "add": True},
        # a prompt scored by the reference policy: logits read once, one number a row
        {"name": "logp_prompt", "op": "logp", "dtype": "bf16", "tokens": 2048, "vocab": 128000, "pad": 0, "back": False},
        # forward and gradient of a short odd batch in fp32
        {"name": "logp_odd", "op": "logp", "dtype": "f32", "tokens": 301, "vocab": 10007, "pad": 1, "back": True},
        # the policy's update on a full batch
        {"name": "policy_batch", "op": "policy", "dtype": "bf16", "tokens": 8192, "vocab": 32000, "pad": 0, "ref": True},
        # a few tokens over an odd vocabulary, rows that no vector load fits
        {"name": "policy_odd", "op": "policy", "dtype": "f16", "tokens": 77, "vocab": 50257, "pad": 0, "ref": False},
        # eight pairs of answers of different lengths
        {"name": "pairs_batch", "op": "pairs", "dtype": "bf16", "pairs": 8, "longest": 512, "vocab": 32000, "pad": 0},
        # one pair of short answers
        {"name": "pairs_one", "op": "pairs", "dtype": "bf16", "pairs": 1, "longest": 9, "vocab": 8192, "pad": 0},
        # a deep stack of narrow layers, fp32 weights that start anywhere in the flat vector
        {"name": "adamw_many", "op": "adamw", "dtype": "f32", "bits": 32, "layers": 40, "cols": 250, "hidden": 701, "vocab": 4001, "align": 1},
        # a wide stack: bf16 weights with fp32 masters, states in 8 bits
        {"name": "adamw_wide", "op": "adamw", "dtype": "bf16", "bits": 8, "layers": 3, "cols": 2048, "hidden": 5632, "vocab": 32000, "align": 128},
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

    op = rng.choice(["embed", "embed_grad", "embed_grad", "logp", "policy", "policy", "pairs", "adamw", "adamw"])
    case = {"op": op, "dtype": rng.choice(["bf16", "f16", "bf16", "f32"])}
    if op == "adamw":
        bits = rng.choice([8, 32])
        case |= {"bits": bits, "cols": size(64, 1024), "hidden": size(64, 2816), "vocab": size(256, 16384),
                 "align": 128 if bits == 8 else rng.choice([1, 8, 128])}
        case["layers"] = size(1, max(1, min(40, 2 ** 26 // (3 * case["cols"] * case["hidden"]))))
        return case
    case["pad"] = rng.choice([0, 0, 1, 5, 8])
    if op in ("embed", "embed_grad"):
        case |= {"tokens": size(1, 16384), "vocab": size(256, 32000), "cols": size(64, 2048)}
        if op == "embed_grad":
            case |= {"wide": rng.random() < 0.6, "add": rng.random() < 0.4}
        return case
    case["vocab"] = size(128, 131072)
    most = max(1, 2 ** 27 // case["vocab"])
    if op == "pairs":
        case["pairs"] = rng.randint(1, 24)
        case["longest"] = size(2, max(3, min(1024, most // (2 * case["pairs"]))))
        return case
    case["tokens"] = size(1, min(8192, most))
    if op == "logp":
        case["back"] = rng.random() < 0.5
    else:
        case["ref"] = rng.random() < 0.6
    return case


def _lengths(case):
    """The lengths of the sequences of a preference batch, chosen and rejected in turn: between a third of the longest and all of it."""
    n, longest = 2 * case["pairs"], case["longest"]
    least = max(1, longest // 3)
    return [longest if i == 0 else least + (i * 2654435761 % 4294967296) * (longest - least) // 4294967296 for i in range(n)]


def _rows(case):
    """Rows of logits: the sequences', and for several pairs a few of padding behind the last one."""
    return case["tokens"] if case["op"] != "pairs" else sum(_lengths(case)) + (5 if case["pairs"] > 1 else 0)


def _sizes(case):
    """The tensors of a stack: (entries, decays) of each."""
    k, f = case["cols"], case["hidden"]
    return [(case["vocab"] * k, False)] + [(k, False), (f * k, True), (f * k, True), (k * f, True)] * case["layers"]


def work(case):
    """The least a pass has to read, write and compute."""
    size = 4 if case["dtype"] == "f32" else 2
    if case["op"] == "adamw":
        n = sum(s for s, _ in _sizes(case))
        # gradient read; weights (16 bits: written, and the fp32 master read and written); two states read and written
        weights = 8 if size == 4 else 10
        states = 16 if case["bits"] == 32 else 4 + 4 / _BLOCK
        return {"bytes": n * (4 + weights + states), "flops": 16 * n}
    if case["op"] == "embed":
        t, k = case["tokens"], case["cols"]
        return {"bytes": t * (8 + 2 * k * size), "flops": t * k}
    if case["op"] == "embed_grad":
        t, k, out = case["tokens"], case["cols"], 4 if case["wide"] else size
        # without a gradient to add to, every row of the table's is written; else the rows of the tokens at hand, at most
        rows = 2 * min(t, case["vocab"]) if case["add"] else case["vocab"]
        return {"bytes": t * (8 + k * size) + rows * k * out, "flops": t * k}
    t, v = _rows(case), case["vocab"]
    if case["op"] == "logp" and not case["back"]:
        return {"bytes": t * (v * size + 16), "flops": 4 * t * v}
    return {"bytes": t * (2 * v * size + 32), "flops": 8 * t * v}


# ---------------------------------------------------------------------------------------------- inputs

def _matrix(gen, rows, cols, pad, dtype, scale=1.0):
    """A matrix whose rows lie cols + pad entries apart."""
    m = torch.randn((rows, cols + pad), generator=gen, device="cuda", dtype=torch.float32)
    return m.mul_(scale).to(dtype)[:, :cols]


def _tokens(gen, n, vocab, padding):
    """Tokens as text has them: the k-th most frequent one about 1 / k as often as the first; a part of them padding (-1)."""
    u = torch.rand(n, generator=gen, device="cuda", dtype=torch.float64)
    t = (torch.exp(u * math.log(vocab + 1.0)).long() - 1).clamp_(0, vocab - 1)
    gone = torch.rand(n, generator=gen, device="cuda") < padding
    return torch.where(gone, torch.full_like(t, -1), t)


def _prepare_adamw(case, gen, s):
    at, n_all, starts = 0, 0, []
    for n, _ in _sizes(case):
        starts.append(at)
        at += -(-n // case["align"]) * case["align"]
    n_all, sizes = at, [n for n, _ in _sizes(case)]
    dtype = _DTYPES[case["dtype"]]
    spread = torch.randn(n_all, generator=gen, device="cuda").mul_(1.5).exp_().mul_(1e-3)   # sizes of the gradient's entries
    g = torch.randn(n_all, generator=gen, device="cuda").mul_(spread)
    m = torch.randn(n_all, generator=gen, device="cuda").mul_(spread).mul_(0.3)
    root = torch.rand(n_all, generator=gen, device="cuda").add_(0.5).mul_(spread)
    p = torch.randn(n_all, generator=gen, device="cuda").mul_(0.02)
    sized = torch.tensor(sizes, device="cuda")
    held = torch.tensor([b - a for a, b in zip(starts, starts[1:] + [n_all])], device="cuda")
    which = torch.arange(len(sizes), device="cuda").repeat_interleave(held)
    within = torch.arange(n_all, device="cuda") - torch.tensor(starts, device="cuda").repeat_interleave(held)
    real = within < sized.repeat_interleave(held)
    g, m, root, p = (x.mul_(real) for x in (g, m, root, p))        # between the tensors: zeros
    s |= {"step": 100, "lr": 3e-4, "seed": int(torch.randint(0, 2 ** 31, (1,), generator=gen, device="cuda")), "grad": g}
    s["wd"] = [0.1 if decays else 0.0 for _, decays in _sizes(case)]
    s["decay"] = torch.tensor(s["wd"], device="cuda", dtype=torch.float64).repeat_interleave(held)
    s["which"], s["within"] = which, within
    s["p"], s["master"] = p.to(dtype), (None if dtype == torch.float32 else p)
    if case["bits"] == 8:
        s["mq"], s["me"] = _nearest(m)
        s["vq"], s["ve"] = _nearest(root)
    else:
        s["m"], s["v"] = m, root.square_()

    def pieces(x, block=1):
        return [x[a // block: a // block + -(-n // block)] for a, n in zip(starts, sizes)]

    # the tensors of the model: slices of the flat vectors
    s["params"], s["grads"] = pieces(s["p"]), pieces(g)
    s["masters"] = None if s["master"] is None else pieces(s["master"])
    if case["bits"] == 8:
        s["ms"] = list(zip(pieces(s["mq"]), pieces(s["me"], _BLOCK)))
        s["vs"] = list(zip(pieces(s["vq"]), pieces(s["ve"], _BLOCK)))
    else:
        s["ms"], s["vs"] = pieces(s["m"]), pieces(s["v"])
    return s


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(int(seed))
    s = {"case": dict(case)}
    if case["op"] == "adamw":
        return _prepare_adamw(case, gen, s)
    dtype, pad = _DTYPES[case["dtype"]], case["pad"]
    if case["op"] in ("embed", "embed_grad"):
        t, v, k = case["tokens"], case["vocab"], case["cols"]
        s["scale"] = math.sqrt(k)
        s["tokens"] = _tokens(gen, t, v, 0.0 if t < 64 else 0.1)
        if case["op"] == "embed":
            s["w"] = _matrix(gen, v, k, pad, dtype, 1.0 / math.sqrt(k))
            return s
        s["dy"] = _matrix(gen, t, k, pad, dtype)
        out = torch.float32 if case["wide"] else dtype
        # without `add` the gradient's buffer has whatever was there
        s["dw"] = _matrix(gen, v, k, pad, out, 0.1)
        return s
    t, v = _rows(case), case["vocab"]
    z = _matrix(gen, t, v, pad, dtype, 2.5)
    s["z"] = z
    # chosen tokens: mostly likely ones; some rows have none (prompts, padding)
    y = torch.where(torch.rand(t, generator=gen, device="cuda") < 0.3, torch.randint(0, v, (t,), generator=gen, device="cuda"), z.argmax(1))
    if t >= 8:
        y = torch.where(torch.rand(t, generator=gen, device="cuda") < 0.1, torch.full_like(y, -1), y)
    s["y"], s["scale"] = y, 1.0 / 0.8
    if case["op"] == "logp":
        if case["back"]:
            s["dlogp"] = torch.randn(t, generator=gen, device="cuda") / t
        return s
    logp, _ = _logp64(s)
    if case["op"] == "policy":
        off = 0.2 * torch.randn(t, generator=gen, device="cuda", dtype=torch.float64)
        # a ratio within fp32's error of a border would be a matter of rounding: none lies nearer than 1e-4
        for edge in (math.log(1.0 - _CLIP_LOW), math.log(1.0 + _CLIP_HIGH)):
            off = torch.where((off - edge).abs() < 1e-4, off + 1e-3, off)
        s["old"] = (logp - off).float()
        s["advantage"] = torch.randn(t, generator=gen, device="cuda") + 0.2
        s["weight"] = torch.where(y < 0, 0.0, 1.0 / max(1, int((y >= 0).sum()))).float()
        s["ref"] = (logp + 0.3 * torch.randn(t, generator=gen, device="cuda", dtype=torch.float64)).float() if case["ref"] else None
        return s
    ends = torch.tensor([0] + _lengths(case), device="cuda").cumsum(0)
    s["offsets"] = ends.to(torch.int32)
    counted = torch.cat([logp.new_zeros(1), torch.where(y < 0, 0.0, logp).cumsum(0)])
    total = counted[ends[1:]] - counted[ends[:-1]]
    s["reference"] = (total + 5.0 * torch.randn(total.shape, generator=gen, device="cuda", dtype=torch.float64)).float()
    return s


# ---------------------------------------------------------------------------------------------- plain forms

def _softmax_parts(z, scale):
    """exp(scale z - largest), their sums and the largest entries of fp32 rows."""
    z = z.float() * scale
    top = z.amax(1, keepdim=True)
    e = torch.exp(z - top)
    return z, e, e.sum(1, keepdim=True), top


def _plain_logp(s):
    z, e, total, top = _softmax_parts(s["z"], s["scale"])
    y = s["y"]
    lse = (torch.log(total.double()) + top.double())[:, 0]
    chosen = z.gather(1, y.clamp(min=0)[:, None])[:, 0].double()
    return torch.where(y < 0, 0.0, chosen - lse), lse, e, total


def _plain_dz(s, coef, e, total):
    """scale coef (1[j = y] - softmax), rows without a chosen token zero."""
    y = s["y"]
    coef = torch.where(y < 0, 0.0, coef).float()[:, None] * s["scale"]
    dz = e.mul_(-coef / total)
    dz.scatter_add_(1, y.clamp(min=0)[:, None], coef)
    return dz.to(s["z"].dtype)


def _logp64(s):
    """The log-probabilities of the chosen tokens in 64 bits (zero where there is none), and the rows' log-sum-exp."""
    z = s["z"].double() * s["scale"]
    lse = torch.logsumexp(z, 1)
    y = s["y"]
    return torch.where(y < 0, 0.0, z.gather(1, y.clamp(min=0)[:, None])[:, 0] - lse), lse


def _scales(x):
    """Exponents e of the power-of-two scales: the smallest with amax <= 448 * 2^e in each block."""
    n = -(-x.numel() // _BLOCK)
    a = torch.nn.functional.pad(x.abs(), (0, n * _BLOCK - x.numel())).reshape(n, _BLOCK)
    top = a.amax(1)
    m, e = torch.frexp(top)
    return torch.where(top > 0, torch.where(m <= 0.875, e - 9, e - 8), -126).clamp(min=-126)


def _powers(e):
    return torch.ldexp(torch.ones_like(e, dtype=torch.float32), e).to(torch.float8_e8m0fnu)


def _nearest(x):
    """The 8-bit form, rounded to nearest."""
    e = _scales(x)
    return torch.ldexp(x, -e.repeat_interleave(_BLOCK)[: x.numel()]).to(torch.float8_e4m3fn), _powers(e)


def _taken(q, e):
    return q.float() * e.float().repeat_interleave(_BLOCK)[: q.numel()]


def _mix(x):
    """32 bits mixed into 32 bits (int64 tensors)."""
    x = x ^ (x >> 16)
    x = (x * 0x85EBCA6B) & 0xFFFFFFFF
    x = x ^ (x >> 13)
    x = (x * 0xC2B2AE35) & 0xFFFFFFFF
    return x ^ (x >> 16)


def _random(s):
    """16 random bits an entry for each state, from the seed, the step, the tensor's number and the entry's."""
    start = _mix(torch.full_like(s["which"], (s["seed"] + 0x9E3779B9 * s["step"]) & 0xFFFFFFFF))
    h = _mix(_mix((start + s["which"]) & 0xFFFFFFFF) ^ s["within"])
    return h & 0xFFFF, h >> 16


def _at_random(x, bits, keep_positive):
    """The 8-bit form, rounded up in size with the probability that the rest bears to a step."""
    e = _scales(x)
    wide = e.repeat_interleave(_BLOCK)[: x.numel()]
    a = torch.ldexp(x.abs(), -wide)
    small = a < 2.0 ** -6                          # below it the steps are 2^-9 wide, as between 2^-6 and 2^-5
    b = torch.where(small, a + 2.0 ** -6, a).view(torch.int32) + (bits << 4).int()
    b = (b & -0x100000).view(torch.float32)
    b = torch.where(small, b - 2.0 ** -6, b)
    if keep_positive:
        b = torch.where((a > 0) & (b == 0), 2.0 ** -9, b)
    return torch.copysign(b, x).to(torch.float8_e4m3fn), _powers(e)


def _plain_adamw(s):
    c = s["case"]
    g = s["grad"]
    eight = c["bits"] == 8
    m = _taken(s["mq"], s["me"]) if eight else s["m"]
    v = _taken(s["vq"], s["ve"]).square() if eight else s["v"]
    p = s["p"] if s["master"] is None else s["master"]
    m = _BETA1 * m + (1.0 - _BETA1) * g
    v = _BETA2 * v + (1.0 - _BETA2) * (g * g)
    root = torch.sqrt(v)
    c1, c2 = 1.0 - _BETA1 ** s["step"], 1.0 - _BETA2 ** s["step"]
    new = p - s["lr"] * (s["decay"].float() * p + (m / c1) / (root / math.sqrt(c2) + _EPS))
    out = {"p": s["p"].copy_(new)}
    if s["master"] is not None:
        out["master"] = s["master"].copy_(new)
    if eight:
        rm, rv = _random(s)
        for name, (q, e) in (("m", _at_random(m, rm, False)), ("v", _at_random(root, rv, True))):
            out[name + "q"], out[name + "e"] = s[name + "q"].copy_(q), s[name + "e"].copy_(e)
    else:
        out["m"], out["v"] = s["m"].copy_(m), s["v"].copy_(v)
    s["step"] += 1
    return out


def _plain(s):
    c = s["case"]
    if c["op"] == "adamw":
        return _plain_adamw(s)
    if c["op"] == "embed":
        t = s["tokens"]
        return {"y": (s["w"][t.clamp(min=0)].float() * s["scale"] * (t >= 0)[:, None]).to(s["w"].dtype)}
    if c["op"] == "embed_grad":
        t = s["tokens"]
        sums = torch.zeros(s["dw"].shape, device=t.device)
        sums.index_add_(0, t.clamp(min=0), s["dy"].float() * (t >= 0)[:, None])
        sums *= s["scale"]
        return {"dw": s["dw"].copy_(sums + s["dw"].float() if c["add"] else sums)}
    logp, lse, e, total = _plain_logp(s)
    if c["op"] == "logp":
        out = {"logp": logp.float(), "lse": lse.float()}
        if c["back"]:
            out["dz"] = _plain_dz(s, s["dlogp"], e, total)
        return out
    if c["op"] == "policy":
        w, a = s["weight"].double(), s["advantage"].double()
        r = torch.exp(logp - s["old"].double())
        free, held = r * a, r.clamp(1.0 - _CLIP_LOW, 1.0 + _CLIP_HIGH) * a
        clipped = free > held
        pg = -torch.minimum(free, held)
        slope = torch.where(clipped, 0.0, -free)
        d = torch.zeros_like(logp) if s["ref"] is None else s["ref"].double() - logp
        kl = torch.expm1(d) - d
        slope = slope - _KL * torch.expm1(d)
        sums = torch.stack([(w * (pg + _KL * kl)).sum(), (w * pg).sum(), (w * kl).sum(), (w * clipped).sum()])
        return {"stats": sums.float(), "logp": logp.float(), "dz": _plain_dz(s, w * slope, e, total)}
    ends = s["offsets"].long()
    upto = torch.cat([logp.new_zeros(1), logp.cumsum(0)])
    sums = upto[ends[1:]] - upto[ends[:-1]]
    ahead = sums - s["reference"].double()
    h = _PAIR_BETA * (ahead[0::2] - ahead[1::2])
    loss = ((1.0 - _SMOOTH) * torch.log1p(torch.exp(-h)) + _SMOOTH * torch.log1p(torch.exp(h))).mean()
    dh = _PAIR_BETA / h.numel() * (_SMOOTH - 1.0 / (1.0 + torch.exp(h)))
    which = torch.arange(sums.numel(), device=h.device).repeat_interleave(ends[1:] - ends[:-1], output_size=sum(_lengths(c)))
    coef = torch.stack([dh, -dh], 1).reshape(-1)[which]
    coef = torch.nn.functional.pad(coef, (0, logp.numel() - coef.numel()))
    return {"loss": loss.float()[None], "margin": h.float(), "sums": sums.float(), "dz": _plain_dz(s, coef, e, total)}


# ---------------------------------------------------------------------------------------------- the framework's calls

def _own(s):
    import paper_1907_12205_b200 as dx
    c = s["case"]
    if c["op"] == "adamw":
        dx.detox_adamw(s["params"], s["grads"], s["ms"], s["vs"], s["step"], s["lr"], beta1=_BETA1, beta2=_BETA2, eps=_EPS,
                       weight_decay=s["wd"], masters=s["masters"], seed=s["seed"])
        s["step"] += 1
        return {k: s[k] for k in ("p", "master", "m", "v", "mq", "me", "vq", "ve") if s.get(k) is not None}
    if c["op"] == "embed":
        return {"y": dx.detox_embedding(s["tokens"], s["w"], scale=s["scale"])}
    if c["op"] == "embed_grad":
        return {"dw": dx.detox_embedding_backward(s["dy"], s["tokens"], c["vocab"], scale=s["scale"], dw=s["dw"], accumulate=c["add"])}
    if c["op"] == "logp":
        logp, lse = dx.detox_token_logp(s["z"], s["y"], scale=s["scale"])
        out = {"logp": logp, "lse": lse}
        if c["back"]:
            out["dz"] = dx.detox_token_logp_backward(s["dlogp"], s["z"], s["y"], lse, scale=s["scale"])
        return out
    if c["op"] == "policy":
        r = dx.detox_policy_loss(s["z"], s["y"], s["old"], s["advantage"], ref_logp=s["ref"], weight=s["weight"], clip_low=_CLIP_LOW,
                                 clip_high=_CLIP_HIGH, kl_coef=_KL, scale=s["scale"])
        return {"stats": r.stats, "logp": r.logp, "dz": r.dz}
    r = dx.detox_preference_loss(s["z"], s["y"], s["offsets"], s["reference"], beta=_PAIR_BETA, smoothing=_SMOOTH, scale=s["scale"])
    return {"loss": r.loss, "margin": r.margin, "sums": r.sums, "dz": r.dz}


def run(state):
    return _own(state) if own else _plain(state)


# ---------------------------------------------------------------------------------------------- 64 bits

def exact(case, seed):
    """The definitions in 64 bits, on the inputs of this seed."""
    s = prepare(case, seed)
    op = case["op"]
    if op == "adamw":
        return _exact_adamw(case, s)
    if op == "embed":
        y = s["w"].double().index_select(0, s["tokens"].clamp(min=0)) * s["scale"]
        y[s["tokens"] < 0] = 0.0
        return {"y": y}
    if op == "embed_grad":
        keep = s["tokens"] >= 0
        dw = s["dw"].double() if case["add"] else torch.zeros(s["dw"].shape, dtype=torch.float64, device="cuda")
        return {"dw": dw.index_put((s["tokens"][keep],), s["scale"] * s["dy"][keep].double(), accumulate=True)}
    z, y = s["z"].double() * s["scale"], s["y"]
    there = torch.nonzero(y >= 0)[:, 0]
    logs = torch.log_softmax(z, 1)
    lse = (z - logs)[:, 0]
    logp = torch.zeros(y.shape, dtype=torch.float64, device="cuda")
    logp[there] = logs[there, y[there]]
    del z

    def slope_of_rows(coef):
        """The gradient of sum coef logp."""
        dz = -torch.exp(logs)
        dz[there, y[there]] += 1.0
        return dz * (coef * (y >= 0))[:, None] * s["scale"]

    if op == "logp":
        out = {"logp": logp, "lse": lse}
        return out | {"dz": slope_of_rows(s["dlogp"].double())} if case["back"] else out
    if op == "policy":
        w, a, old = s["weight"].double(), s["advantage"].double(), s["old"].double()
        ratio = torch.exp(logp - old)
        low, high = 1.0 - _CLIP_LOW, 1.0 + _CLIP_HIGH
        clipped = torch.where(a > 0, ratio > high, (ratio < low) & (a < 0))
        pg = -a * torch.where(clipped, torch.where(a > 0, high, low), ratio)
        coef = torch.where(clipped, 0.0, -a * ratio)
        kl = torch.zeros_like(logp)
        if s["ref"] is not None:
            gap = s["ref"].double() - logp
            kl = torch.exp(gap) - gap - 1.0
            coef = coef + _KL * (1.0 - torch.exp(gap))
        stats = torch.stack([torch.dot(w, pg) + _KL * torch.dot(w, kl), torch.dot(w, pg), torch.dot(w, kl), w[clipped].sum()])
        return {"stats": stats, "logp": logp, "dz": slope_of_rows(w * coef)}
    lengths = _lengths(case)
    parts = torch.split(logp[: sum(lengths)], lengths)
    sums = torch.stack([p.sum() for p in parts])
    lead = (sums - s["reference"].double()).view(-1, 2)
    h = _PAIR_BETA * (lead[:, 0] - lead[:, 1])
    loss = -(1.0 - _SMOOTH) * torch.nn.functional.logsigmoid(h) - _SMOOTH * torch.nn.functional.logsigmoid(-h)
    dh = (-(1.0 - _SMOOTH) * torch.sigmoid(-h) + _SMOOTH * torch.sigmoid(h)) * _PAIR_BETA / case["pairs"]
    coef = torch.zeros_like(logp)
    at = 0
    for i, n in enumerate(lengths):
        coef[at: at + n] = dh[i // 2] * (1.0 if i % 2 == 0 else -1.0)
        at += n
    return {"loss": loss.mean()[None], "margin": h, "sums": sums, "dz": slope_of_rows(coef)}


def _exact_adamw(case, s):
    eight = case["bits"] == 8
    g = s["grad"].double()

    def state(name):
        q, e = s[name + "q"].double(), s[name + "e"].double()
        return (q.reshape(-1, _BLOCK) * e[:, None]).reshape(-1)

    m = state("m") if eight else s["m"].double()
    v = state("v") ** 2 if eight else s["v"].double()
    p = (s["p"] if s["master"] is None else s["master"]).double()
    m, v = m + (1.0 - _BETA1) * (g - m), v + (1.0 - _BETA2) * (g ** 2 - v)
    t = s["step"]
    direction = m / -math.expm1(t * math.log(_BETA1)) / (torch.sqrt(v / -math.expm1(t * math.log(_BETA2))) + _EPS)
    new = p * (1.0 - s["lr"] * s["decay"]) - s["lr"] * direction
    out = {"p": new}
    if s["master"] is not None:
        out["master"] = new
    if not eight:
        return out | {"m": m, "v": v}

    def rounded(x, bits, positive):
        """Values and scales; a step is 2^-3 of the power of two below the value, 2^-9 at least."""
        b = x.reshape(-1, _BLOCK)
        top = b.abs().amax(1, keepdim=True)
        e = torch.ceil(torch.log2(torch.clamp(top, min=1e-300) / 448.0))
        e = torch.where(top > 448.0 * torch.exp2(e), e + 1, e)
        e = torch.where(top <= 448.0 * torch.exp2(e - 1), e - 1, e).clamp(min=-126)
        a = b.abs() / torch.exp2(e)
        step = torch.exp2(torch.floor(torch.log2(torch.clamp(a, min=2.0 ** -6))) - 3)
        q = torch.floor(a / step + bits.reshape(b.shape).double() / 65536.0) * step
        if positive:
            q = torch.where((a > 0) & (q == 0), 2.0 ** -9, q)
        return (q * torch.sign(b)).reshape(-1), torch.exp2(e)[:, 0]

    def mixed(x):
        x = (x ^ (x >> 16)) * 0x85EBCA6B % 2 ** 32
        x = (x ^ (x >> 13)) * 0xC2B2AE35 % 2 ** 32
        return x ^ (x >> 16)

    first = mixed((s["seed"] + 0x9E3779B9 * t) % 2 ** 32)
    h = mixed(mixed((first + s["which"]) % 2 ** 32) ^ s["within"])
    out["mq"], out["me"] = rounded(m, h % 65536, False)
    out["vq"], out["ve"] = rounded(torch.sqrt(v), h // 65536, True)
    return out
