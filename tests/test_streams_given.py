"""The aggregation's functions on a stream that is given to the call, while the current stream is busy with memory of its own."""
import numpy as np
import pytest
import torch

import paper_1907_12205_b200 as dx
from paper_1907_12205_b200 import binding

DEV = "cuda:0"
N, R, D = 15, 3, 20_000
NAP = 100_000_000          # clocks: some fifty milliseconds


def calls():
    gen = torch.Generator(device=DEV).manual_seed(0)
    votes = torch.randn((N // R, D), generator=gen, device=DEV)
    X = votes.repeat_interleave(R, 0).contiguous()
    members = np.arange(N, dtype=np.int32)
    members_dev = torch.arange(N, dtype=torch.int32, device=DEV)
    sets, ids = [0, 2, 5], np.arange(5)
    pipe = dx.Pipeline(N, R, D, members, dx.AGG_MEAN, sets, ids, dx.AGG_COORD_MEDIAN)
    torch.cuda.synchronize()
    return {
        "vote": lambda **k: dx.detox_vote(X, R, members, **k),
        "hier_mean": lambda **k: dx.detox_hier_mean(votes, sets, ids, **k),
        "vote_hier_mean": lambda **k: dx.detox_vote_hier_mean(X, R, members, sets, ids, **k),
        "many": lambda **k: dx.detox_vote_hier_mean_many(X[:, :100], R, members_dev, sets, **k),
        "median": lambda **k: dx.agg_coord_median(X, **k),
        "trimmed": lambda **k: dx.agg_trimmed_mean(X, 2, **k),
        "sign": lambda **k: dx.agg_sign_majority(X, **k),
        "geometric": lambda **k: dx.agg_geometric_median(X, 4, **k),
        "distances": lambda **k: dx.agg_pairwise_sqdist(X, **k),
        "multikrum": lambda **k: dx.agg_multikrum(X, 2, 5, **k),
        "bulyan": lambda **k: dx.agg_bulyan(X, 2, **k),
        "pipeline": lambda **k: [t for t in dx.detox_aggregate(pipe, X, **k).values() if t is not None],
    }


def tensors(r):
    return [t for t in (r if isinstance(r, (tuple, list)) else (r,)) if t is not None]


@pytest.mark.gpu
@pytest.mark.parametrize("as_handle", [False, True])
@pytest.mark.parametrize("name", ["vote", "hier_mean", "vote_hier_mean", "many", "median", "trimmed", "sign", "geometric", "distances",
                                  "multikrum", "bulyan", "pipeline"])
def test_outputs_do_not_take_memory_that_the_current_stream_still_writes(name, as_handle):
    call = calls()[name]
    want = [t.clone() for t in tensors(call())]
    side, before = torch.cuda.Stream(), torch.cuda.current_stream()
    torch.cuda.synchronize()
    blocks = [torch.empty(s.untyped_storage().nbytes(), dtype=torch.uint8, device=DEV) for s in tensors(call()) for _ in range(3)]
    torch.cuda.synchronize()
    torch.cuda._sleep(NAP)
    for b in blocks:
        b.fill_(0x5A)
    del blocks, b
    got = tensors(call(stream=side.cuda_stream if as_handle else side))
    assert torch.cuda.current_stream() == before
    torch.cuda.synchronize()
    assert len(got) == len(want) and all(torch.equal(a, b) for a, b in zip(got, want))


@pytest.mark.gpu
def test_a_stream_may_be_given_by_its_place_and_the_default_one_by_its_handle():
    X = torch.randn((7, 1000), generator=torch.Generator(device=DEV).manual_seed(1), device=DEV)
    want = dx.agg_coord_median(X)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    got = dx.agg_coord_median(X, None, None, side)
    side.synchronize()
    assert torch.equal(got, want)
    with torch.cuda.stream(side):
        got = dx.agg_coord_median(X, None, None, 0)
        assert torch.cuda.current_stream() == side
    torch.cuda.synchronize()
    assert torch.equal(got, want)


def test_the_functions_keep_their_signatures():
    import inspect
    assert list(inspect.signature(binding.detox_vote).parameters) == ["X", "r", "members", "Z", "winner", "want_Z", "ws", "stream"]
    assert binding.detox_vote.__doc__.startswith("Majority vote")


def test_a_workspace_elsewhere_or_smaller_than_it_looks_is_refused():
    host, meta = torch.device("cpu"), torch.device("meta")
    t = torch.empty(512, dtype=torch.uint8)
    assert binding._ws(300, t, host)[1:] == (t.data_ptr(), 512)
    for where in (torch.device(DEV), meta):
        with pytest.raises(TypeError, match="ws"):
            binding._ws(300, t, where)
    for wrong in (t[:1].expand(512), t[::2]):
        with pytest.raises(ValueError, match="ws"):
            binding._ws(300, wrong, host)
