"""The gradients of the gated products asked for one at a time, which the C interface allows: the same bits as all of them together."""
import ctypes

import pytest
import torch

import paper_1907_12205_b200 as dx

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF16, F32 = torch.bfloat16, torch.float32


@pytest.mark.parametrize("eight", [False, True])
@pytest.mark.parametrize("kept", [False, True])
@pytest.mark.parametrize("tokens,in_dim,hidden", [(3, 640, 200), (300, 72, 264), (2300, 1024, 1920)])
def test_only_dx_or_only_the_weight_gradients(tokens, in_dim, hidden, kept, eight):
    gen = torch.Generator(device=DEV).manual_seed(tokens)
    shapes = ((tokens, in_dim), (hidden, in_dim), (hidden, in_dim), (tokens, hidden))
    x, wg, wu, dh = (torch.randn(s, generator=gen, device=DEV).to(BF16) for s in shapes)
    pair = dx.detox_checkpoint_pack(x)
    k = dx.detox_gated(x, wg, wu, keep=True)[1] if kept else None
    want = dx.detox_gated_backward(dh, pair if eight else x, wg, wu, kept=k, dw_dtype=F32)
    d = dx.GatedDesc(dtype=dx.DTYPE_BFLOAT, act=dx.ACT_SILU, tokens=tokens, in_dim=in_dim, hidden=hidden, Wg=wg.data_ptr(), ldwg=in_dim,
                     Wu=wu.data_ptr(), ldwu=in_dim)
    if eight:
        d.XQ, d.ldxq, d.XE, d.ldxe = pair[0].data_ptr(), pair[0].stride(0), pair[1].data_ptr(), pair[1].stride(0)
    else:
        d.X, d.ldx = x.data_ptr(), in_dim
    if kept:
        d.GQ, d.GE, d.UQ, d.UE = k.gq.data_ptr(), k.ge.data_ptr(), k.uq.data_ptr(), k.ue.data_ptr()
        d.ldq, d.lde = k.gq.stride(0), k.ge.stride(0)
    lib = dx.load()
    need = lib.detox_gated_backward_workspace_bytes(ctypes.byref(d))
    for with_dx, with_dw in ((True, False), (False, True), (True, True)):
        ws = torch.full((need,), 0x5A, dtype=torch.uint8, device=DEV)      # (the status word, too)
        gx = torch.full((tokens, in_dim), 7.0, dtype=BF16, device=DEV)
        a, b = (torch.full((hidden, in_dim), 7.0, device=DEV) for _ in range(2))
        st = lib.detox_gated_backward(ctypes.byref(d), dh.data_ptr(), hidden, gx.data_ptr() if with_dx else None, in_dim if with_dx else 0,
                                      a.data_ptr() if with_dw else None, b.data_ptr() if with_dw else None, in_dim if with_dw else 0,
                                      dx.DTYPE_FLOAT, ws.data_ptr(), need, torch.cuda.current_stream().cuda_stream)
        assert st == 0 and dx.read_status(ws) == 0
        assert torch.equal(gx, want[0]) if with_dx else bool((gx == 7.0).all())
        for got, ref in ((a, want[1]), (b, want[2])):
            assert torch.equal(got, ref) if with_dw else bool((got == 7.0).all())
