"""What the worker-side operators refuse, before anything is launched (no GPU needed: pointers are fake and never read)."""
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
ODD = ctypes.c_void_p(0x10001)


@pytest.fixture(scope="module")
def lib():
    from paper_1907_12205_b200 import build
    build.build()
    return dx.load()


def test_codes_and_descriptor_match_the_header():
    codes = {n: int(v) for n, v in re.findall(r"\b(DETOX_(?:DTYPE|ACT)_[A-Z]+)\s*=\s*(\d+)", HEADER)}
    assert codes == {"DETOX_DTYPE_FLOAT": dx.DTYPE_FLOAT, "DETOX_DTYPE_HALF": dx.DTYPE_HALF, "DETOX_DTYPE_BFLOAT": dx.DTYPE_BFLOAT,
                     "DETOX_ACT_SILU": dx.ACT_SILU, "DETOX_ACT_GELU": dx.ACT_GELU, "DETOX_ACT_RELU": dx.ACT_RELU}
    assert int(re.search(r"#define DETOX_KEEP_BLOCK (\d+)", HEADER).group(1)) == dx.KEEP_BLOCK
    body = re.search(r"typedef struct \{((?:(?!typedef struct).)*?)\} detox_gated_desc;", HEADER, re.S).group(1)
    body = re.sub(r"/\*.*?\*/", "", body, flags=re.S)
    names = [n.strip(" *") for line in re.findall(r"([^;]+);", body) for n in re.sub(r"^\s*(const )?\w+\*? ", "", line.strip()).split(",")]
    assert names == [f[0] for f in dx.GatedDesc._fields_]
    assert ctypes.sizeof(dx.GatedDesc) == 160


def test_checkpoint_refusals(lib):
    pack = lib.detox_checkpoint_pack
    assert pack(3, P, 64, 4, 64, P, 64, P, 1, None) == BAD              # no such type
    assert pack(2, P, 64, -1, 64, P, 64, P, 1, None) == BAD
    assert pack(2, P, 64, 4, 0, P, 64, P, 1, None) == BAD
    assert pack(2, P, 63, 4, 64, P, 64, P, 1, None) == BAD              # rows overlap
    assert pack(2, P, 64, 4, 64, P, 63, P, 1, None) == BAD
    assert pack(2, P, 129, 4, 129, P, 129, P, 1, None) == BAD           # two scales a row
    assert pack(2, None, 64, 4, 64, P, 64, P, 1, None) == BAD
    assert pack(2, ODD, 64, 4, 64, P, 64, P, 1, None) == BAD            # not aligned to its entries
    assert pack(2, P, 64, 4, 64, P, 64, None, 1, None) == BAD
    assert pack(2, P, 64, (1 << 30) + 1, 64, P, 64, P, 1, None) == UNSUPPORTED
    assert pack(2, None, 64, 0, 64, None, 64, None, 1, None) == 0       # no rows: nothing to do
    unpack = lib.detox_checkpoint_unpack
    assert unpack(2, P, 64, P, 1, 4, 64, P, 63, None) == BAD
    assert unpack(2, None, 64, P, 1, 4, 64, P, 64, None) == BAD
    assert unpack(7, P, 64, P, 1, 4, 64, P, 64, None) == BAD
    assert unpack(2, P, 64, P, 1, 4, 64, ODD, 64, None) == BAD
    assert unpack(2, None, 64, None, 1, 0, 64, None, 64, None) == 0


def test_norm_refusals(lib):
    def norm(dtype=2, X=P, ldx=64, R=None, ldr=0, w=P, rows=4, cols=64, eps=1e-6, S=None, lds=0, Y=P, ldy=64, Q=None, ldq=0, E=None,
             lde=0, rstd=None):
        return lib.detox_rmsnorm(dtype, X, ldx, R, ldr, w, rows, cols, eps, S, lds, Y, ldy, Q, ldq, E, lde, rstd, None)

    assert norm(dtype=9) == BAD and norm(X=None) == BAD and norm(w=None) == BAD and norm(ldx=63) == BAD and norm(ldy=63) == BAD
    assert norm(eps=-1.0) == BAD and norm(eps=float("nan")) == BAD
    assert norm(Y=None) == BAD                                           # nothing asked for
    assert norm(R=P, ldr=63) == BAD and norm(S=P, lds=63) == BAD and norm(X=ODD) == BAD
    assert norm(Q=P, ldq=64) == BAD and norm(E=P, lde=1) == BAD          # values without scales, scales without values
    assert norm(rows=-1) == BAD and norm(cols=0) == BAD
    assert norm(cols=32769, ldx=32769, ldy=32769) == UNSUPPORTED
    assert norm(rows=0, X=None) == 0

    def back(dtype=2, dY=P, lddy=64, dS=None, ldds=0, S=P, lds=64, w=P, rstd=P, rows=4, cols=64, dX=P, lddx=64, dw=P, ws=P, wb=1 << 20):
        return lib.detox_rmsnorm_backward(dtype, dY, lddy, dS, ldds, S, lds, w, rstd, rows, cols, dX, lddx, dw, ws, wb, None)

    assert back(dtype=-1) == BAD and back(dY=None) == BAD and back(S=None) == BAD and back(rstd=None) == BAD and back(lddx=5) == BAD
    assert back(dX=None, dw=None) == BAD and back(dS=P, ldds=3) == BAD
    assert back(ws=None) == WORKSPACE and back(wb=16) == WORKSPACE and back(ws=ctypes.c_void_p(0x10010)) == WORKSPACE
    assert back(cols=40000, lddy=40000, lds=40000, lddx=40000) == UNSUPPORTED
    assert lib.detox_rmsnorm_backward_workspace_bytes(10, 40000) == 0
    assert lib.detox_rmsnorm_backward_workspace_bytes(-1, 4) == 0
    assert lib.detox_rmsnorm_backward_workspace_bytes(8192, 2048) >= 2048 * 4


def desc(**kw):
    d = binding.GatedDesc(dtype=2, act=0, tokens=4, in_dim=64, hidden=128, X=0x10000, ldx=64, Wg=0x20000, ldwg=64, Wu=0x30000, ldwu=64)
    for k, v in kw.items():
        setattr(d, k, v)
    return d


def test_gated_refusals(lib):
    def size(**kw):
        return lib.detox_gated_workspace_bytes(ctypes.byref(desc(**kw)))

    def fwd(H=P, ldh=128, ws=P, wb=1 << 30, **kw):
        return lib.detox_gated(ctypes.byref(desc(**kw)), H, ldh, ws, wb, None)

    assert size() >= 4 and fwd(ws=None) == WORKSPACE and fwd(wb=0) == WORKSPACE and fwd(ws=ctypes.c_void_p(0x10010)) == WORKSPACE
    for bad in (dict(act=3), dict(act=-1), dict(dtype=5), dict(tokens=-1), dict(in_dim=0), dict(hidden=0), dict(X=None), dict(ldx=63),
                dict(ldwg=63), dict(Wu=None), dict(Wg=0x20001), dict(X=0x10001), dict(GQ=0x40000), dict(GQ=0x40000, GE=0x50000),
                dict(GQ=0x40000, GE=0x50000, UQ=0x60000, UE=0x70000, ldq=127, lde=1),
                dict(GQ=0x40000, GE=0x50000, UQ=0x60000, UE=0x70000, ldq=128, lde=0),
                dict(X=None, XQ=0x40000, ldxq=64), dict(X=None, XQ=0x40000, ldxq=63, XE=0x50000, ldxe=1)):
        assert fwd(**bad) == BAD and size(**bad) == 0, bad
    assert fwd(dtype=0) == UNSUPPORTED and fwd(tokens=(1 << 30) + 1) == UNSUPPORTED
    assert fwd(H=None) == BAD and fwd(ldh=127) == BAD and lib.detox_gated(None, P, 128, P, 1 << 20, None) == BAD
    # an input that TMA cannot address, or one in 8 bits, is laid out again in the workspace
    assert size(ldx=65) > size() and size(X=None, XQ=0x40000, ldxq=64, XE=0x50000, ldxe=1) > size() and size(Wg=0x20002) > size()

    def back(dH=P, lddh=128, dX=P, lddx=64, dWg=P, dWu=P, lddw=64, dw=2, ws=P, wb=1 << 30, **kw):
        return lib.detox_gated_backward(ctypes.byref(desc(**kw)), dH, lddh, dX, lddx, dWg, dWu, lddw, dw, ws, wb, None)

    assert back(dH=None) == BAD and back(lddh=127) == BAD and back(lddx=63) == BAD and back(lddw=63) == BAD and back(dw=1) == BAD
    assert back(dWg=None) == BAD and back(dX=None, dWg=None, dWu=None) == BAD and back(act=9) == BAD
    assert back(ws=None) == WORKSPACE and back(wb=64) == WORKSPACE
    assert lib.detox_gated_backward_workspace_bytes(ctypes.byref(desc())) >= 2 * 4 * 128 * 2


def test_the_binding_checks_types_before_the_library_is_asked():
    x = torch.zeros((4, 8))
    with pytest.raises(TypeError):
        dx.detox_checkpoint_pack(x)                    # not on the GPU
    with pytest.raises(TypeError):
        dx.detox_rmsnorm(x, torch.ones(8))
    with pytest.raises(TypeError):
        dx.detox_gated(x, x, x)
