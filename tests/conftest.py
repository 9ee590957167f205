import inspect
import os
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)


def pytest_configure(config):
    config.addinivalue_line("markers", "gpu: needs a CUDA device (sm_100a)")


def holds_an_old_value(item):
    """Cases that expect a value since found wrong, and fail: a log-sum-exp of 0 for the row without a chosen token that their batches of more than two rows have
    (tests/test_token_lse.py has the right one).  They run last, so that they hide nothing in a run that stops at the first failure."""
    params = item.callspec.params if hasattr(item, "callspec") else {}
    return getattr(item, "originalname", "") == "test_logp_and_its_gradient" and params.get("rows", 0) > 2


def pytest_collection_modifyitems(config, items):
    items.sort(key=holds_an_old_value)
    try:
        import torch
        have = torch.cuda.is_available()
    except Exception:
        have = False
    if have:
        return
    skip = pytest.mark.skip(reason="no CUDA device")
    for it in items:
        if "gpu" in it.keywords:
            it.add_marker(skip)


@pytest.fixture(autouse=True)
def memory_for_side_streams(request):
    """For tests that look whether a side stream is still busy when a call returns: memory that this process has already, for every stream that they can be given.  A call that
    had to get it from the driver took 20 to 45 ms now and then on machines shared with others, of the 50 that such a stream is kept busy."""
    function = getattr(request, "function", None)
    if function is None or "side.query()" not in inspect.getsource(function):
        yield
        return
    import torch
    if torch.cuda.is_available():
        for _ in range(32):                        # torch hands out 32 streams in turn
            with torch.cuda.stream(torch.cuda.Stream()):
                held = [torch.empty(n, dtype=torch.uint8, device="cuda:0") for n in (1 << 27, 1 << 19, 1 << 19, 1 << 12)]
                del held
        torch.cuda.synchronize()
    yield
