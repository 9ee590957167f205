"""The least eps of the optimizer's step, and what is below it (no GPU needed)."""
import os
import re

import pytest

import paper_1907_12205_b200 as dx

HEADER = open(os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include", "detox.h")).read()


def test_what_is_below_the_least_eps_is_refused():
    least, least8 = (float(re.search(r"#define DETOX_ADAMW_LEAST_EPS%s (\S+)" % n, HEADER).group(1)) for n in ("", "_8"))
    assert least == 1e-18 and least8 == 1e-15
    dx.detox_adamw([], [], [], [], 1, 1e-3, eps=least)
    for eps in (least * 0.99, 1e-25, 1e-38, 1e-46, 5e-324):
        with pytest.raises(dx.DetoxError):
            dx.detox_adamw([], [], [], [], 1, 1e-3, eps=eps)
