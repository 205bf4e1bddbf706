"""The example that runs clipping, detection and the clipped update together:
the loss falls although two of seven workers send -100 times their
gradients, which every iteration finds."""
import importlib.util
import os

import pytest

from _helpers import device

pytestmark = pytest.mark.gpu

PATH = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples",
                    "clipped_training.py")


@pytest.mark.parametrize("optimizer", ["sgd", "adamw"])
def test_clipped_training(optimizer):
    spec = importlib.util.spec_from_file_location("clipped_training", PATH)
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    losses, found = example.train(30, optimizer, device())
    assert losses[-1] < 0.5 * losses[0]
    assert all(f == frozenset(example.ADVERSARIES) for f in found)
