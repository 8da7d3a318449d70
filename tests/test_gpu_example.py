"""The example runs every operator in the loop that it is meant for, and learns."""
import math
import os
import sys

import pytest

pytestmark = pytest.mark.gpu
sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


def test_text_classifier_learns():
    import train_text_classifier as example
    losses = example.train(steps=60, workers=5)
    assert all(math.isfinite(v) for v in losses)
    assert abs(losses[0] - math.log(example.CLASSES)) < 0.3         # chance at the start
    assert sum(losses[-5:]) / 5 < 0.5 * math.log(example.CLASSES)
    assert example.train(steps=3, workers=5) == losses[:3]          # the same again: no result depends on the run
