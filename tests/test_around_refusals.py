"""What the embedding, the losses over logits and the optimizer's step refuse, before anything is launched (no GPU needed: pointers are
fake and never read)."""
import ctypes
import os
import re

import pytest
import torch

import paper_1907_12205_b200 as dx
from paper_1907_12205_b200 import binding

HEADER = open(os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include", "detox.h")).read()
BAD, UNSUPPORTED, WORKSPACE = 1, 2, 3
P = ctypes.c_void_p(0x10000)
Q = ctypes.c_void_p(0x20000)
ODD = ctypes.c_void_p(0x10001)
NAN, INF = float("nan"), float("inf")


@pytest.fixture(scope="module")
def lib():
    from paper_1907_12205_b200 import build
    build.build()
    return dx.load()


@pytest.mark.parametrize("name,mirror,size", [
    ("detox_policy_desc", binding.PolicyDesc, 104), ("detox_preference_desc", binding.PreferenceDesc, 88),
    ("detox_adamw_tensor", binding.AdamWTensor, 80), ("detox_adamw_desc", binding.AdamWDesc, 72)])
def test_structures_match_the_header(name, mirror, size):
    body = re.search(r"typedef struct \{((?:(?!typedef struct).)*?)\} %s;" % name, HEADER, re.S).group(1)
    body = re.sub(r"/\*.*?\*/", "", body, flags=re.S)
    names = [n.strip(" *") for line in re.findall(r"([^;]+);", body) for n in re.sub(r"^\s*(const )?\w+\*? ", "", line.strip()).split(",")]
    assert names == [f[0] for f in mirror._fields_]
    assert ctypes.sizeof(mirror) == size


def test_codes_match_the_header():
    codes = {n: int(v) for n, v in re.findall(r"\b(DETOX_INDEX_[A-Z0-9]+)\s*=\s*(\d+)", HEADER)}
    assert codes == {"DETOX_INDEX_INT32": 0, "DETOX_INDEX_INT64": 1}
    assert int(re.search(r"#define DETOX_LOGITS_MAX_COLS (\d+)", HEADER).group(1)) == dx.LOGITS_MAX_COLS


def test_embedding(lib):
    def look(dtype=2, W=P, ldw=64, vocab=10, cols=64, index=1, tokens=P, rows=4, Y=Q, ldy=64):
        return lib.detox_embedding(dtype, W, ldw, vocab, cols, index, tokens, rows, 1.0, Y, ldy, None)

    for bad in (dict(dtype=3), dict(index=2), dict(index=-1), dict(W=None), dict(W=ODD), dict(ldw=63), dict(vocab=0), dict(cols=0),
                dict(rows=-1), dict(tokens=None), dict(tokens=ctypes.c_void_p(0x10004)), dict(Y=None), dict(ldy=63)):
        assert look(**bad) == BAD, bad
    assert look(vocab=(1 << 30) + 1) == UNSUPPORTED and look(rows=(1 << 30) + 1) == UNSUPPORTED
    assert look(rows=0, W=None, tokens=None, Y=None) == 0

    def back(dtype=2, dY=P, lddy=64, index=0, tokens=P, rows=4, vocab=10, cols=64, dW=Q, lddw=64, dw=0, add=0, ws=P, wb=1 << 30):
        return lib.detox_embedding_backward(dtype, dY, lddy, index, tokens, rows, vocab, cols, 1.0, dW, lddw, dw, add, ws, wb, None)

    for bad in (dict(dtype=-1), dict(index=2), dict(dY=None), dict(lddy=63), dict(tokens=None), dict(tokens=ctypes.c_void_p(0x10002)),
                dict(rows=-1), dict(vocab=0), dict(vocab=-5), dict(cols=0), dict(dW=None), dict(lddw=63), dict(dw=1), dict(dw=7),
                dict(dW=ctypes.c_void_p(0x20002))):
        assert back(**bad) == BAD, bad
    assert back(ws=None) == WORKSPACE and back(wb=100) == WORKSPACE and back(ws=ctypes.c_void_p(0x10010)) == WORKSPACE
    assert back(vocab=(1 << 30) + 1) == UNSUPPORTED
    assert back(rows=0, dY=None, tokens=None, add=1) == 0                # nothing to add
    size = lib.detox_embedding_backward_workspace_bytes
    assert size(-1, 4, 4) == 0 and size(4, 0, 4) == 0 and size(4, 4, 0) == 0 and size(1000, 500, 64) > 8 * 1000 + 4 * 500


def test_token_logp(lib):
    def logp(dtype=2, Z=P, ldz=64, rows=4, vocab=64, index=1, y=P, scale=1.0, out=Q, lse=Q):
        return lib.detox_token_logp(dtype, Z, ldz, rows, vocab, index, y, scale, out, lse, None)

    for bad in (dict(dtype=3), dict(Z=None), dict(Z=ODD), dict(ldz=63), dict(rows=-1), dict(vocab=0), dict(index=5), dict(y=None),
                dict(scale=0.0), dict(scale=-1.0), dict(scale=NAN), dict(scale=INF), dict(out=None, lse=None), dict(out=ODD), dict(lse=ODD)):
        assert logp(**bad) == BAD, bad
    assert logp(vocab=dx.LOGITS_MAX_COLS + 1, ldz=1 << 20) == UNSUPPORTED
    assert logp(rows=0, Z=None, y=None, out=None, lse=None) == 0

    def back(dtype=2, Z=P, ldz=64, rows=4, vocab=64, index=1, y=P, scale=1.0, lse=Q, dlogp=Q, dZ=Q, lddz=64):
        return lib.detox_token_logp_backward(dtype, Z, ldz, rows, vocab, index, y, scale, lse, dlogp, dZ, lddz, None)

    for bad in (dict(dtype=9), dict(lse=None), dict(dlogp=None), dict(dlogp=ODD), dict(dZ=None), dict(lddz=63), dict(scale=-2.0),
                dict(dZ=P, lddz=72)):                                    # in place, but with other rows
        assert back(**bad) == BAD, bad
    assert back(rows=0, Z=None, y=None, lse=None, dlogp=None, dZ=None) == 0


def policy_desc(**kw):
    d = binding.PolicyDesc(dtype=2, index=1, rows=4, vocab=64, Z=0x10000, ldz=64, y=0x10000, old_logp=0x10000, advantage=0x10000,
                           clip_low=0.2, clip_high=0.2, kl_coef=0.1, scale=1.0, grad_scale=1.0)
    for k, v in kw.items():
        setattr(d, k, v)
    return d


def test_policy_loss(lib):
    def loss(stats=Q, logp=None, dZ=Q, lddz=64, ws=P, wb=1 << 20, **kw):
        return lib.detox_policy_loss(ctypes.byref(policy_desc(**kw)), stats, logp, dZ, lddz, ws, wb, None)

    for bad in (dict(dtype=4), dict(index=2), dict(rows=-1), dict(vocab=0), dict(Z=None), dict(ldz=8), dict(y=None), dict(old_logp=None),
                dict(advantage=None), dict(old_logp=0x10002), dict(ref_logp=0x10001), dict(weight=0x10002), dict(clip_low=-0.1),
                dict(clip_low=1.5), dict(clip_low=NAN), dict(clip_high=-0.1), dict(clip_high=INF), dict(kl_coef=NAN), dict(scale=0.0),
                dict(grad_scale=INF), dict(stats=None), dict(stats=ODD), dict(logp=ODD), dict(lddz=63), dict(dZ=P, lddz=80)):
        assert loss(**bad) == BAD, bad
    assert loss(vocab=dx.LOGITS_MAX_COLS + 1, ldz=1 << 20) == UNSUPPORTED
    assert loss(ws=None) == WORKSPACE and loss(wb=8) == WORKSPACE and loss(ws=ctypes.c_void_p(0x10020)) == WORKSPACE
    assert lib.detox_policy_loss(None, Q, None, Q, 64, P, 1 << 20, None) == BAD
    assert lib.detox_policy_loss_workspace_bytes(-1) == 0 and lib.detox_policy_loss_workspace_bytes(1 << 20) >= 32 * 148


def preference_desc(**kw):
    d = binding.PreferenceDesc(dtype=2, index=0, rows=4, vocab=64, pairs=1, Z=0x10000, ldz=64, y=0x10000, offsets=0x10000, ref=0x10000,
                               beta=0.1, smoothing=0.0, scale=1.0, grad_scale=1.0)
    for k, v in kw.items():
        setattr(d, k, v)
    return d


def test_preference_loss(lib):
    def loss(out=Q, margin=Q, sums=Q, dZ=Q, lddz=64, ws=P, wb=1 << 20, **kw):
        return lib.detox_preference_loss(ctypes.byref(preference_desc(**kw)), out, margin, sums, dZ, lddz, ws, wb, None)

    for bad in (dict(dtype=4), dict(pairs=-1), dict(offsets=None), dict(offsets=0x10002), dict(ref=None), dict(beta=NAN), dict(smoothing=-0.1),
                dict(smoothing=1.1), dict(smoothing=NAN), dict(grad_scale=NAN), dict(scale=-1.0), dict(out=None), dict(margin=None),
                dict(sums=None), dict(lddz=63), dict(dZ=P, lddz=72), dict(Z=None), dict(y=None)):
        assert loss(**bad) == BAD, bad
    assert loss(pairs=1 << 30) == UNSUPPORTED and loss(vocab=dx.LOGITS_MAX_COLS + 1, ldz=1 << 20) == UNSUPPORTED
    assert loss(ws=None) == WORKSPACE and loss(wb=64) == WORKSPACE
    assert lib.detox_preference_loss(None, Q, Q, Q, Q, 64, P, 1 << 20, None) == BAD
    size = lib.detox_preference_loss_workspace_bytes
    assert size(-1, 1) == 0 and size(1, -1) == 0 and size(100, 7) >= 3 * 400 + 56


def adamw(lib, bits=32, desc=(), count=1, null=False, **kw):
    t = binding.AdamWTensor(P=0x10000, G=0x20000, master=None, M=0x30000, ME=0x31000, V=0x40000, VE=0x41000, n=100, p_dtype=0, g_dtype=0)
    for k, v in kw.items():
        setattr(t, k, v)
    d = binding.AdamWDesc(bits=bits, lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8, grad_scale=1.0, step=1)
    for k, v in dict(desc).items():
        setattr(d, k, v)
    return lib.detox_adamw(ctypes.byref(d), None if null else ctypes.byref(t), count, None)


def test_adamw(lib):
    for bad in (dict(lr=NAN), dict(lr=INF), dict(beta1=1.0), dict(beta1=-0.1), dict(beta2=1.0), dict(beta2=NAN), dict(eps=0.0), dict(eps=-1e-8),
                dict(eps=INF), dict(step=0), dict(step=-3), dict(grad_scale=NAN), dict(lr_dev=0x10002), dict(step_dev=0x10004)):
        assert adamw(lib, desc=bad) == BAD, bad
    for bad in (dict(n=-1), dict(p_dtype=3), dict(g_dtype=-1), dict(P=None), dict(G=None), dict(M=None), dict(V=None), dict(P=0x10002),
                dict(G=0x20001), dict(M=0x30002), dict(V=0x40001), dict(G=0x10000), dict(V=0x30000), dict(weight_decay=NAN),
                dict(p_dtype=2, master=0x50002), dict(p_dtype=2, master=0x20000)):
        assert adamw(lib, **bad) == BAD, bad
    assert adamw(lib, bits=16) == BAD and adamw(lib, bits=8, ME=None) == BAD and adamw(lib, bits=8, VE=None) == BAD
    assert adamw(lib, master=0x50000) == UNSUPPORTED                     # fp32 weights are their own master
    assert adamw(lib, p_dtype=2, g_dtype=1) == UNSUPPORTED and adamw(lib, p_dtype=1, g_dtype=2) == UNSUPPORTED
    assert adamw(lib, n=1 << 41) == UNSUPPORTED
    assert adamw(lib, count=-1) == BAD and adamw(lib, null=True) == BAD
    assert adamw(lib, null=True, count=0) == 0 and adamw(lib, n=0, P=None, G=None, M=None, V=None) == 0
    assert lib.detox_adamw(None, None, 0, None) == BAD


def test_the_binding_checks_types_before_the_library_is_asked():
    x, t = torch.zeros((4, 8)), torch.zeros(4, dtype=torch.int64)
    f = torch.zeros(4)
    for call in (lambda: dx.detox_embedding(t, x), lambda: dx.detox_embedding_backward(x, t, 8), lambda: dx.detox_token_logp(x, t),
                 lambda: dx.detox_token_logp_backward(f, x, t, f), lambda: dx.detox_policy_loss(x, t, f, f),
                 lambda: dx.detox_preference_loss(x, t, torch.zeros(3, dtype=torch.int32), torch.zeros(2)),
                 lambda: dx.detox_adamw([x], [x], [x], [x], 1, 1e-3)):
        with pytest.raises(TypeError):
            call()                                                       # not on the GPU
    with pytest.raises(ValueError):
        dx.detox_adamw([x], [], [], [], 1, 1e-3)
    with pytest.raises(ValueError):
        dx.detox_adamw([], [], [], [], 1, 1e-3, weight_decay=[0.1])
    with pytest.raises(ValueError):
        dx.detox_adamw([], [], [], [], 1, 1e-3, seed=1 << 32)
    with pytest.raises(dx.DetoxError):
        dx.detox_adamw([], [], [], [], 0, 1e-3)
    assert dx.detox_adamw([], [], [], [], 1, 1e-3) is None
    with pytest.raises(ValueError):
        dx.detox_adamw_state([x], bits=16)
    m, v = dx.detox_adamw_state([x, torch.zeros(300)], bits=8)
    assert m[1][0].shape == (300,) and v[1][1].shape == (3,) and float(m[0][1].float()[0]) == 2.0 ** -126
