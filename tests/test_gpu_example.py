"""The example that runs the operators and the transfer together: the loss falls towards what the synthetic text
allows, the receivers hold the trainer's BF16 weights and score a batch as the trainer does."""
import math
import os
import sys

import pytest

pytestmark = pytest.mark.gpu


def test_training_with_the_operators_keeps_receivers_in_step():
    sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
    try:
        import train_and_sync
    finally:
        sys.path.pop(0)
    r = train_and_sync.run(steps=30, vocab=512, hidden=128, tokens=2048, say=None)
    assert abs(r["losses"][0] - math.log(512)) < 0.5              # an untrained model: near the uniform loss
    assert r["losses"][-1] < r["losses"][0] - 2.0                 # 30 epochs' worth of a vocabulary of 512 are learnt
    # an element the reconstruction takes for unchanged stays stale: the paper's method allows few of them
    assert r["stale"] <= r["elements"] * 1e-3
    assert abs(r["here"] - r["there"]) <= 2e-3 * r["here"]
