"""The example of a small language model: it learns to count and goes on counting over its cache."""
import importlib.util
import math
import os

import pytest

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_language_model_learns_and_continues():
    spec = importlib.util.spec_from_file_location("language_model", os.path.join(ROOT, "examples", "language_model.py"))
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    losses, share = example.run(steps=80, verbose=False)
    # untrained: about the uniform distribution's log(499); a model that counts right is far below one of the 61 words that occur
    assert abs(losses[0] - math.log(499)) < 1.5
    assert sum(losses[-5:]) / 5 < 0.5 * math.log(61)
    assert share > 0.5
