"""The example that runs sampler, cache, recurrence, loss and optimizer together: it learns."""
import os
import sys

import pytest

pytestmark = pytest.mark.gpu
sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


@pytest.mark.parametrize("bits", [8, 32])
def test_the_example_learns(bits):
    import link_training
    losses, right = link_training.train(steps=60, bits=bits, seed=1)
    # untrained the order is a coin's; users keep to one of eight kinds, so most other items can be told from the true one
    assert sum(right[-10:]) / 10 > 0.7, right[-10:]
    assert sum(losses[-10:]) < 0.9 * sum(losses[:10])
