"""Kernels whose CTAs store to each other's shared memory: a CTA may be written to only once it is known to have started.

The order is checked in the source, for every kernel that does so; on the GPU, the values of rows that clusters of every size share."""
import os
import re

import pytest
import torch

import paper_1907_12205_b200 as dx

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_1907_12205_b200", "csrc")
DEV = "cuda:0"
TYPES = [torch.bfloat16, torch.float16, torch.float32]
U = 2.0 ** -24


def kernels(source):
    """(name, body) of every __global__ function."""
    for m in re.finditer(r"__global__ void[^{;]*?(\w+)\(const __grid_constant__[^{;]*\) \{", source):
        depth, at = 1, m.end()
        while depth:
            depth += {"{": 1, "}": -1}.get(source[at], 0)
            at += 1
        yield m.group(1), source[m.end():at]


def test_a_cluster_has_started_before_its_shared_memory_is_written():
    source = open(os.path.join(CSRC, "token_loss.cu")).read()
    found = {name: body for name, body in kernels(source) if "store_at(" in body}
    assert set(found) == {"policy_kernel", "score_kernel"}
    for name, body in found.items():
        tell, wait, store = (body.index(w) for w in ("cluster_tell_started()", "cluster_wait_started()", "store_at("))
        assert tell < wait < store, name
    # whoever has told waits before it leaves: the way out of rows that are not read does, too (the one before it belongs to kernels without clusters)
    body = found["score_kernel"]
    ways_out = [body[:m.start()].splitlines()[-2:] for m in re.finditer(r"\breturn;", body[:body.index("store_at(")])]
    assert len(ways_out) == 2 and "row >= g.rows" in ways_out[0][-1] and any("cluster_wait_started()" in line for line in ways_out[1])
    assert [f for f in os.listdir(CSRC) if "st.shared::cluster" in open(os.path.join(CSRC, f)).read()] in (["gated.cu", "token_loss.cu"], ["token_loss.cu", "gated.cu"])


def batch(rows, vocab, dtype, pad, gone):
    gen = torch.Generator(device=DEV).manual_seed(rows + vocab)
    z = (3 * torch.randn((rows, vocab + pad), generator=gen, device=DEV)).to(dtype)[:, :vocab]
    y = torch.randint(0, vocab, (rows,), generator=gen, device=DEV)
    y[torch.rand(rows, generator=gen, device=DEV) < gone] = -1
    return z, y


def slack(z):
    """As for the log-probabilities elsewhere: exponents, powers and logarithm, fewer than 100 additions."""
    x = z.double()
    return U * (120 + 6 * (x.amax(1) - x.amin(1)) + 6 * x.abs().amax(1))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,vocab", [(3, 8200), (5, 16390), (2, 32000), (148, 16384), (70, 33000), (36, 65600), (18, 131072), (2, 262144), (1, 75000), (7, 32770)])
@pytest.mark.parametrize("gone", [0.0, 0.5, 1.0])
def test_rows_that_a_cluster_shares(dtype, rows, vocab, gone):
    for pad in (0, 3):
        z, y = batch(rows, vocab, dtype, pad, gone)
        lse = torch.logsumexp(z.double(), 1)
        logp = torch.where(y < 0, 0.0, z.double().gather(1, y.clamp(min=0)[:, None])[:, 0] - lse)
        off = slack(z)
        old, a = (logp + 0.05).float(), torch.ones(rows, device=DEV)
        first = None
        # many calls on the same rows, which then lie in L2: CTAs have their part of a row at very different times
        for _ in range(30):
            got = dx.detox_token_logp(z, y)
            alone = dx.detox_token_logp(z, y, want_lse=False).logp
            pol = dx.detox_policy_loss(z, y, old, a)
            now = (got.logp, got.lse, alone, pol.logp, pol.stats, pol.dz)
            first = first or now
            assert all(torch.equal(p, q) for p, q in zip(now, first))
        assert bool(((got.lse.double() - lse).abs() <= off).all())
        assert all(bool(((x.double() - logp).abs() <= off).all()) for x in (got.logp, alone, pol.logp))
        # the gradient of a row adds up to nothing: its probabilities, each rounded, to 1
        half = torch.finfo(dtype).eps / 2
        tiny = {torch.bfloat16: 0.0, torch.float16: vocab * 2.0 ** -25, torch.float32: 0.0}[dtype]
        want = 2 * (half + 1e-4) / rows + tiny
        assert bool((pol.dz.double().sum(1).abs() <= want * 1.06).all()) and bool((pol.dz[y < 0] == 0).all())
