"""The example's arguments: refused before anything runs on a GPU."""
import os
import sys

import pytest

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
try:
    import train_and_sync as example
finally:
    sys.path.pop(0)


@pytest.mark.parametrize("heads", [1, 2, 3, 6, -4])
def test_heads_that_two_receivers_cannot_share_are_refused(heads, monkeypatch):
    # nothing may be made for such heads, neither weights nor the plan
    monkeypatch.setattr(example.torch, "Generator", lambda *a: pytest.fail("the arguments were taken"))
    with pytest.raises(ValueError, match="multiple of 4"):
        example.run(steps=1, vocab=64, hidden=64, tokens=64, say=None, heads=heads)
