"""The worker-side operators record no graph, and say so: an input that requires grad is refused, except under torch.no_grad()."""
import pytest
import torch

import paper_1907_12205_b200 as dx

BF16 = torch.bfloat16


def arguments(device):
    return {"x": torch.zeros((4, 64), dtype=BF16, device=device), "wg": torch.zeros((32, 64), dtype=BF16, device=device),
            "wu": torch.zeros((32, 64), dtype=BF16, device=device), "dh": torch.zeros((4, 32), dtype=BF16, device=device),
            "w": torch.ones(64, dtype=BF16, device=device), "rstd": torch.ones(4, device=device)}


def calls(t):
    return {"pack": lambda: dx.detox_checkpoint_pack(t["x"]),
            "norm": lambda: dx.detox_rmsnorm(t["x"], t["w"]),
            "norm backward": lambda: dx.detox_rmsnorm_backward(t["x"], t["x"], t["w"], t["rstd"]),
            "gated": lambda: dx.detox_gated(t["x"], t["wg"], t["wu"]),
            "gated backward": lambda: dx.detox_gated_backward(t["dh"], t["x"], t["wg"], t["wu"])}


ARGUMENTS = {"pack": ["x"], "norm": ["x", "w"], "norm backward": ["x", "w", "rstd"], "gated": ["x", "wg", "wu"],
             "gated backward": ["dh", "x", "wg", "wu"]}
CASES = [(c, n) for c, names in ARGUMENTS.items() for n in names]


@pytest.fixture(scope="module", autouse=True)
def built():
    from paper_1907_12205_b200 import build
    build.build()


# the argument that is looked at first: on the host the ones behind it are not reached
@pytest.mark.parametrize("call,name", [("pack", "x"), ("norm", "x"), ("norm backward", "x"), ("gated", "wg"), ("gated backward", "wg")])
def test_refused_in_grad_mode_before_the_device_is_looked_at(call, name):
    t = arguments("cpu")
    t[name].requires_grad_(True)
    with pytest.raises(RuntimeError, match="requires grad"):
        calls(t)[call]()
    with torch.no_grad(), pytest.raises(TypeError):
        calls(t)[call]()


@pytest.mark.gpu
@pytest.mark.parametrize("call,name", CASES)
def test_refused_in_grad_mode_and_taken_without(call, name):
    t = arguments("cuda:0")
    t[name].requires_grad_(True)
    with pytest.raises(RuntimeError, match="requires grad"):
        calls(t)[call]()
    with torch.no_grad():
        out = calls(t)[call]()
    assert not any(r.requires_grad for r in (out if isinstance(out, tuple) else (out,)) if r is not None)
    t[name].requires_grad_(False)
    calls(t)[call]()
