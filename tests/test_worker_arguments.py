"""Arguments that are not what they are taken for: refused, not cut to size."""
import pytest
import torch

import paper_1907_12205_b200 as dx

pytestmark = pytest.mark.gpu
BF16 = torch.bfloat16


def test_an_activation_that_does_not_fit_its_type_is_not_another_one():
    x, w = torch.zeros((8, 64), dtype=BF16, device="cuda:0"), torch.zeros((32, 64), dtype=BF16, device="cuda:0")
    for act in (2 ** 32, 2 ** 32 + dx.ACT_GELU, -2 ** 32):
        with pytest.raises(dx.DetoxError) as e:
            dx.detox_gated(x, w, w, act=act)
        assert e.value.code == 1
    with pytest.raises(OverflowError):
        dx.detox_gated(x, w, w, act=2 ** 70)


def test_a_flag_without_a_truth_value_is_refused():
    x, w = torch.zeros((8, 64), dtype=BF16, device="cuda:0"), torch.zeros((32, 64), dtype=BF16, device="cuda:0")
    both = torch.ones(2, dtype=torch.bool)
    for call in (lambda: dx.detox_gated(x, w, w, keep=both), lambda: dx.detox_rmsnorm(x, w[0], want_y=both),
                 lambda: dx.detox_rmsnorm(x, w[0], want_q=both)):
        with pytest.raises(RuntimeError, match="ambiguous"):
            call()
