"""The example's training step: the operators and the codecs together, on a model that learns."""
import importlib.util
import math
import os

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.mark.gpu
def test_training_step_learns():
    spec = importlib.util.spec_from_file_location("training_step", os.path.join(ROOT, "examples", "training_step.py"))
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    history = example.main(steps=30)
    losses = [loss for loss, _ in history]
    assert all(math.isfinite(v) for pair in history for v in pair)
    # the loss falls to a part of where it started: residual and target differ by a projection that can be learnt
    assert losses[-1] < 0.5 * losses[0] and max(losses[-5:]) < losses[0]
