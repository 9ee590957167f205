"""All tensors of a call lie on one GPU, its workspace among them: anything else is refused before a launch."""
import pytest
import torch

import paper_1907_12205_b200 as dx

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF16 = torch.bfloat16


def tensors(device=DEV):
    return {"x": torch.zeros((8, 64), dtype=BF16, device=device), "wg": torch.zeros((32, 64), dtype=BF16, device=device),
            "wu": torch.zeros((32, 64), dtype=BF16, device=device), "dh": torch.zeros((8, 32), dtype=BF16, device=device),
            "w": torch.zeros(64, dtype=BF16, device=device), "rstd": torch.ones(8, device=device)}


def calls(t, ws=None):
    kept = dx.Kept(torch.zeros((2, 8, 32), dtype=torch.uint8, device=DEV).view(torch.float8_e4m3fn),
                   torch.zeros((2, 8, 1), dtype=torch.uint8, device=DEV).view(torch.float8_e8m0fnu))
    return [lambda: dx.detox_gated(t["x"], t["wg"], t["wu"], ws=ws),
            lambda: dx.detox_gated_backward(t["dh"], t["x"], t["wg"], t["wu"], ws=ws),
            lambda: dx.detox_gated_backward(t["dh"], t["x"], t["wg"], t["wu"], kept=kept, ws=ws),
            lambda: dx.detox_rmsnorm_backward(t["x"], t["x"], t["w"], t["rstd"], ws=ws)]


def test_a_workspace_that_is_not_on_the_gpu_or_smaller_than_it_looks_is_refused():
    t = tensors()
    size = 1 << 20
    for call in calls(t, torch.empty(size, dtype=torch.uint8)):
        with pytest.raises(TypeError, match="ws"):
            call()
    with pytest.raises(TypeError, match="ws"):
        calls(t, 7)[0]()
    for call in calls(t, torch.empty(1, dtype=torch.uint8, device=DEV).expand(size)):   # one byte that says it is a million
        with pytest.raises(ValueError, match="ws"):
            call()
    for call in calls(t, torch.empty(2 * size, dtype=torch.uint8, device=DEV)[::2]):
        with pytest.raises(ValueError, match="ws"):
            call()
    for call in calls(t, torch.empty(size, dtype=torch.uint8, device=DEV)):
        call()


@pytest.mark.parametrize("name", ["x", "wg", "wu", "dh", "w", "rstd"])
def test_a_tensor_on_the_host_is_refused_wherever_it_stands(name):
    t = tensors()
    t[name] = t[name].cpu()
    refused = 0
    for call in calls(t):
        try:
            call()
        except TypeError:
            refused += 1
    assert refused == {"x": 4, "wg": 3, "wu": 3, "dh": 2, "w": 1, "rstd": 1}[name]


@pytest.mark.skipif(torch.cuda.device_count() < 2, reason="needs two GPUs")
@pytest.mark.parametrize("name", ["x", "wg", "wu", "dh", "w", "rstd"])
def test_tensors_of_two_gpus_are_refused(name):
    t = tensors()
    t[name] = t[name].to("cuda:1")
    refused = 0
    for call in calls(t):
        try:
            call()
        except (ValueError, TypeError):
            refused += 1
    assert refused == {"x": 4, "wg": 3, "wu": 3, "dh": 2, "w": 1, "rstd": 1}[name]
    other = torch.empty(1 << 20, dtype=torch.uint8, device="cuda:1")
    for call in calls(tensors(), other):
        with pytest.raises(ValueError, match="ws"):
            call()
