"""The example of redundant workers: their gradients agree bit for bit, the vote drops the attackers, and the loss falls."""
import os
import sys

import pytest

pytestmark = pytest.mark.gpu

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


@pytest.mark.parametrize("tokens,dim,hidden", [(64, 96, 264), (130, 200, 333)])
def test_feed_forward_workers_train(tokens, dim, hidden):
    import feed_forward_workers as example
    losses, equal = example.train(steps=12, tokens=tokens, dim=dim, hidden=hidden, log=None)
    assert equal
    assert losses[-1] < 0.7 * losses[0]
