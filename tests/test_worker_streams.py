"""The worker-side operators on a stream that is given to the call, while the current stream is busy with memory of its own."""
import pytest
import torch

import paper_1907_12205_b200 as dx

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF16, F32 = torch.bfloat16, torch.float32
NAP = 100_000_000          # clocks: some fifty milliseconds


def inputs(tokens, in_dim, hidden):
    gen = torch.Generator(device=DEV).manual_seed(0)
    shapes = ((tokens, in_dim), (hidden, in_dim), (hidden, in_dim), (tokens, hidden))
    x, wg, wu, dh = (torch.randn(s, generator=gen, device=DEV) for s in shapes)
    return x.to(BF16), (wg * in_dim ** -0.5).to(BF16), (wu * in_dim ** -0.5).to(BF16), dh.to(BF16)


def calls():
    x, wg, wu, dh = inputs(1000, 512, 768)
    w = wg[0].contiguous()
    n = dx.detox_rmsnorm(x, w, x, want_q=True)
    _, kept = dx.detox_gated(x, wg, wu, keep=True)
    torch.cuda.synchronize()
    flat = lambda r: [t for t in (r if isinstance(r, tuple) else (r,)) if t is not None]  # noqa: E731
    return {
        "pack": lambda **k: flat(dx.detox_checkpoint_pack(x, **k)),
        "unpack": lambda **k: flat(dx.detox_checkpoint_unpack(n.q, n.e, **k)),
        "norm": lambda **k: flat(dx.detox_rmsnorm(x, w, x, want_q=True, **k)),
        "norm backward": lambda **k: flat(dx.detox_rmsnorm_backward(x, n.sum, w, n.rstd, **k)),
        "gated": lambda **k: flat(dx.detox_gated(x, wg, wu, **k)),
        "gated, kept": lambda **k: (lambda r: [r[0], *r[1]])(dx.detox_gated(x, wg, wu, keep=True, **k)),
        "gated backward": lambda **k: flat(dx.detox_gated_backward(dh, x, wg, wu, kept=kept, dw_dtype=F32, **k)),
    }


NAMES = ["pack", "unpack", "norm", "norm backward", "gated", "gated, kept", "gated backward"]


def as_bytes(t):
    return t if t.dtype in (F32, BF16) else t.view(torch.uint8)


@pytest.mark.parametrize("as_handle", [False, True])
@pytest.mark.parametrize("name", NAMES)
def test_outputs_do_not_take_memory_that_the_current_stream_still_writes(name, as_handle):
    """The current stream's pool is full of freed blocks of the outputs' sizes that it is still going to write."""
    call = calls()[name]
    want = [t.clone() for t in call()]
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    blocks = [torch.empty(s.untyped_storage().nbytes(), dtype=torch.uint8, device=DEV) for s in call() for _ in range(3)]
    torch.cuda.synchronize()
    torch.cuda._sleep(NAP)
    for b in blocks:
        b.fill_(0x5A)
    del blocks, b
    got = call(stream=side.cuda_stream if as_handle else side)
    torch.cuda.synchronize()
    assert len(got) == len(want) and all(torch.equal(as_bytes(a), as_bytes(b)) for a, b in zip(got, want))


def test_the_workspace_is_not_handed_out_again_while_the_stream_uses_it():
    x, wg, wu, dh = inputs(8192, 1024, 2048)
    _, kept = dx.detox_gated(x, wg, wu, keep=True)
    want = [t.clone() for t in dx.detox_gated_backward(dh, x, wg, wu, kept=kept)]
    size = dx.detox_gated_backward_workspace_bytes(x, wg, wu, kept=kept)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    for _ in range(5):
        torch.cuda.empty_cache()
        got = dx.detox_gated_backward(dh, x, wg, wu, kept=kept, stream=side)
        for _ in range(20):                       # as long as the products take
            torch.empty(size, dtype=torch.uint8, device=DEV).fill_(0xFF)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_a_given_stream_is_where_the_work_runs_and_the_current_one_stays():
    call = calls()["gated"]
    want = call()[0].clone()
    side, before = torch.cuda.Stream(), torch.cuda.current_stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        torch.cuda._sleep(NAP)
    got = call(stream=side)[0]
    assert torch.cuda.current_stream() == before
    before.synchronize()
    assert not side.query()                       # still behind the nap
    side.synchronize()
    assert torch.equal(got, want)
    with torch.cuda.stream(side):                 # the default stream's handle, from another current stream
        got = call(stream=torch.cuda.default_stream())[0]
        assert torch.cuda.current_stream() == side
    torch.cuda.synchronize()
    assert torch.equal(got, want)
