"""The policy loss of a few wide rows, whose number decides how many CTAs share one: the same results whichever it is."""
import pytest
import torch

import paper_1907_12205_b200 as dx

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
U = 2.0 ** -24


@pytest.mark.parametrize("vocab", [33000, 40001, 50257, 65544, 65541, 131072])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_rows_do_not_depend_on_how_many_there_are(dtype, vocab):
    """Alone a row has a cluster of eight CTAs; 37 .. 148 of them have the sizes between.  The sum's order changes: fewer than 100 additions on either side."""
    most = 149
    gen = torch.Generator(device=DEV).manual_seed(vocab)
    z = (2 * torch.randn((most, vocab), generator=gen, device=DEV)).to(dtype)
    y = torch.randint(0, vocab, (most,), generator=gen, device=DEV)
    logp = torch.log_softmax(z[:4].double(), 1).gather(1, y[:4, None])[:, 0]
    old = torch.full((most,), -10.0, device=DEV)
    one, w = torch.ones(most, device=DEV), torch.full((most,), 0.125, device=DEV)
    want = None
    for rows in (1, 18, 19, 37, 38, 73, 74, 75, 77, 92, 93, 110, 147, 148, 149):
        got = dx.detox_policy_loss(z[:rows], y[:rows], old[:rows], one[:rows], old[:rows], w[:rows], clip_high=1e6, kl_coef=0.1)
        n = min(rows, 4)
        assert bool(((got.logp[:n].double() - logp[:n]).abs() <= U * (200 + 8 * 20)).all())
        want = got.dz[:1].clone() if want is None else want
        off = torch.finfo(dtype).eps + 400 * U
        assert bool(((got.dz[:1].double() - want.double()).abs() <= off * want.double().abs() + 2.0 ** -126).all())
        assert bool(got.dz.isfinite().all())
