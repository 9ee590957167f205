"""The embedding, the losses and the optimizer's step on a stream that is given to the call, on tensors in the wrong place, and captured."""
import pytest
import torch

import paper_1907_12205_b200 as dx

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF16, F32 = torch.bfloat16, torch.float32
NAP = 100_000_000          # clocks: some fifty milliseconds


def inputs(rows=700, vocab=2048, cols=512, device=DEV):
    gen = torch.Generator(device=DEV).manual_seed(0)
    t = {"z": torch.randn((rows, vocab), generator=gen, device=DEV).to(BF16), "y": torch.randint(0, vocab, (rows,), generator=gen, device=DEV),
         "w": torch.randn((vocab, cols), generator=gen, device=DEV).to(BF16), "d": torch.randn((rows, cols), generator=gen, device=DEV).to(BF16),
         "f": torch.randn(rows, generator=gen, device=DEV), "o": torch.tensor([0, 100, 350, 600, 690], dtype=torch.int32, device=DEV),
         "r": torch.full((4,), -900.0, device=DEV)}
    return {k: v.to(device) for k, v in t.items()}


def calls(t, **more):
    flat = lambda r: [x for x in (r if isinstance(r, tuple) else (r,)) if x is not None]  # noqa: E731
    lse = dx.detox_token_logp(t["z"], t["y"]).lse if t["z"].is_cuda else t["f"]
    return {
        "embedding": lambda **k: flat(dx.detox_embedding(t["y"], t["w"], **k)),
        "embedding backward": lambda **k: flat(dx.detox_embedding_backward(t["d"], t["y"], 2048, dw_dtype=F32, **k)),
        "logp": lambda **k: flat(dx.detox_token_logp(t["z"], t["y"], **k)),
        "logp backward": lambda **k: flat(dx.detox_token_logp_backward(t["f"], t["z"], t["y"], lse, **k)),
        "policy": lambda **k: flat(dx.detox_policy_loss(t["z"], t["y"], t["f"] - 8, t["f"], t["f"] - 8, kl_coef=0.1, **k)),
        "preference": lambda **k: flat(dx.detox_preference_loss(t["z"], t["y"], t["o"], t["r"], **k)),
    }


NAMES = ["embedding", "embedding backward", "logp", "logp backward", "policy", "preference"]
WITH_WORKSPACE = ["embedding backward", "policy", "preference"]


def same(got, want):
    as_bits = lambda x: x.contiguous().view(torch.uint8)  # noqa: E731
    return len(got) == len(want) and all(torch.equal(as_bits(a), as_bits(b)) for a, b in zip(got, want))


@pytest.mark.parametrize("as_handle", [False, True])
@pytest.mark.parametrize("name", NAMES)
def test_outputs_and_workspaces_do_not_take_memory_that_the_current_stream_still_writes(name, as_handle):
    """The current stream's pool is full of freed blocks of the outputs' sizes (and of small ones, as workspaces are) that it is still going to write."""
    call = calls(inputs())[name]
    want = [t.clone() for t in call()]
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    sizes = [s.untyped_storage().nbytes() for s in call()] + [256, 4096, 16384, 65536]
    blocks = [torch.empty(n, dtype=torch.uint8, device=DEV) for n in sizes for _ in range(3)]
    torch.cuda.synchronize()
    torch.cuda._sleep(NAP)
    for b in blocks:
        b.fill_(0x5A)
    del blocks, b
    got = call(stream=side.cuda_stream if as_handle else side)
    torch.cuda.synchronize()
    assert same(got, want)


@pytest.mark.parametrize("name", NAMES)
def test_a_given_stream_is_where_the_work_runs(name):
    call = calls(inputs())[name]
    want = [t.clone() for t in call()]
    side, before = torch.cuda.Stream(), torch.cuda.current_stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        torch.cuda._sleep(NAP)
    got = call(stream=side)
    assert torch.cuda.current_stream() == before and not side.query()
    side.synchronize()
    assert same(got, want)


def test_the_optimizer_on_a_given_stream():
    gen = torch.Generator(device=DEV).manual_seed(1)
    p, g = torch.randn(5000, generator=gen, device=DEV), torch.randn(5000, generator=gen, device=DEV)
    want, (m, v) = p.clone(), dx.detox_adamw_state([p])
    dx.detox_adamw([want], [g], m, v, 1, 0.1)
    m, v = dx.detox_adamw_state([p])
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        torch.cuda._sleep(NAP)
    dx.detox_adamw([p], [g], m, v, 1, 0.1, stream=side)
    assert not side.query()
    side.synchronize()
    assert torch.equal(p, want)


@pytest.mark.parametrize("name", NAMES)
def test_captured_and_replayed_on_new_inputs(name):
    t = inputs()
    call = calls(t)[name]
    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = call()
    for seed in range(3):
        gen = torch.Generator(device=DEV).manual_seed(10 + seed)
        t["y"].copy_(torch.randint(-1, 2048, (700,), generator=gen, device=DEV))
        t["z"].copy_(torch.randn((700, 2048), generator=gen, device=DEV))
        t["d"].copy_(torch.randn((700, 512), generator=gen, device=DEV))
        t["f"].copy_(torch.randn(700, generator=gen, device=DEV))
        graph.replay()
        graph.replay()                             # (twice: counters and workspaces start again)
        torch.cuda.synchronize()
        assert same(got, call())


@pytest.mark.parametrize("name", WITH_WORKSPACE)
def test_calls_one_after_another_share_a_workspace(name):
    t, u = inputs(), inputs(rows=690)
    size = max(dx.detox_embedding_backward_workspace_bytes(700, 2048, 512), dx.detox_policy_loss_workspace_bytes(700),
               dx.detox_preference_loss_workspace_bytes(700, 2))
    ws = torch.full((size,), 0xFF, dtype=torch.uint8, device=DEV)
    first, second = calls(t)[name], calls(u)[name]
    want = [[x.clone() for x in f()] for f in (first, second)]
    for _ in range(20):
        got = [first(ws=ws), second(ws=ws)]
        assert same(got[0], want[0]) and same(got[1], want[1])


def test_many_calls_give_the_same_bits():
    t = inputs()
    for name in NAMES:
        call = calls(t)[name]
        want = [x.clone() for x in call()]
        for _ in range(50):
            assert same(call(), want), name


@pytest.mark.parametrize("name", WITH_WORKSPACE)
def test_a_workspace_that_is_not_on_the_gpu_or_too_small_is_refused(name):
    call = calls(inputs())[name]
    with pytest.raises(TypeError, match="ws"):
        call(ws=torch.empty(1 << 24, dtype=torch.uint8))
    with pytest.raises(ValueError, match="ws"):
        call(ws=torch.empty(1, dtype=torch.uint8, device=DEV).expand(1 << 24))
    with pytest.raises(dx.DetoxError):
        call(ws=torch.empty(16, dtype=torch.uint8, device=DEV))
    call(ws=torch.empty(1 << 25, dtype=torch.uint8, device=DEV))


@pytest.mark.parametrize("key,refused", [("z", 4), ("y", 6), ("w", 1), ("d", 1), ("f", 2), ("o", 1), ("r", 1)])
def test_a_tensor_on_the_host_is_refused_wherever_it_stands(key, refused):
    t = inputs()
    good = calls(t)
    lse = dx.detox_token_logp(t["z"], t["y"]).lse
    t[key] = t[key].cpu()
    n = 0
    for name, call in good.items():
        try:
            call()
        except (TypeError, ValueError):
            n += 1
    assert n == refused and lse.is_cuda


def test_shapes_and_types_are_checked():
    t = inputs()
    z, y, f, w, d, o, r = (t[k] for k in "zyfwdor")
    for error, call in (
            (TypeError, lambda: dx.detox_embedding(y.to(torch.int16), w)), (TypeError, lambda: dx.detox_embedding(y[None], w)),
            (TypeError, lambda: dx.detox_embedding(y[::2], w)), (TypeError, lambda: dx.detox_embedding(y, w.double())),
            (ValueError, lambda: dx.detox_embedding(y, w, out=torch.empty((700, 511), dtype=BF16, device=DEV))),
            (TypeError, lambda: dx.detox_embedding(y, w, out=torch.empty((700, 512), device=DEV))),
            (ValueError, lambda: dx.detox_embedding(y, w.T)), (ValueError, lambda: dx.detox_embedding_backward(d, y[:-1], 2048)),
            (ValueError, lambda: dx.detox_embedding_backward(d, y, 0)), (ValueError, lambda: dx.detox_embedding_backward(d, y, 2048, accumulate=True)),
            (ValueError, lambda: dx.detox_embedding_backward(d, y, 2048, dw=torch.empty((2047, 512), device=DEV))),
            (dx.DetoxError, lambda: dx.detox_embedding_backward(d, y, 2048, dw_dtype=torch.float16)),
            (ValueError, lambda: dx.detox_token_logp(z, y[1:])), (TypeError, lambda: dx.detox_token_logp(z, f)),
            (dx.DetoxError, lambda: dx.detox_token_logp(z, y, scale=0.0)), (TypeError, lambda: dx.detox_token_logp_backward(f[1:], z, y, f)),
            (TypeError, lambda: dx.detox_token_logp_backward(f.to(BF16), z, y, f)), (TypeError, lambda: dx.detox_policy_loss(z, y, f[1:], f)),
            (TypeError, lambda: dx.detox_policy_loss(z, y, f, f, ref_logp=f.double())), (TypeError, lambda: dx.detox_policy_loss(z, y, f, f, weight=f[:3])),
            (dx.DetoxError, lambda: dx.detox_policy_loss(z, y, f, f, clip_low=2.0)), (ValueError, lambda: dx.detox_policy_loss(z, y, f, f, want_grad=False, dz=z)),
            (TypeError, lambda: dx.detox_policy_loss(z, y, f, f, dz=z.float())), (TypeError, lambda: dx.detox_preference_loss(z, y, o.long(), r)),
            (TypeError, lambda: dx.detox_preference_loss(z, y, o[1:], r)), (ValueError, lambda: dx.detox_preference_loss(z, y, o, r[:3])),
            (dx.DetoxError, lambda: dx.detox_preference_loss(z, y, o, r, smoothing=1.5))):
        with pytest.raises(error):
            call()
    wide = torch.empty((2, dx.LOGITS_MAX_COLS + 1), dtype=BF16, device=DEV)
    with pytest.raises(dx.DetoxError):
        dx.detox_token_logp(wide, y[:2])
    x = z.detach().clone().requires_grad_()
    with pytest.raises(RuntimeError, match="requires grad"):
        dx.detox_policy_loss(x, y, f, f)


@pytest.mark.skipif(torch.cuda.device_count() < 2, reason="needs two GPUs")
def test_tensors_of_two_gpus_are_refused_and_another_device_than_the_current_one_works():
    t = inputs()
    other = inputs(device="cuda:1")
    for name, call in calls(other).items():
        assert same([x.cpu() for x in call()], [x.cpu() for x in calls(t)[name]()])
    with pytest.raises(ValueError):
        dx.detox_embedding(other["y"], t["w"])
    with pytest.raises(ValueError):
        dx.detox_policy_loss(t["z"], t["y"], other["f"], t["f"])
