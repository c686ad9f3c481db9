"""The example runs the token operators together as a training loop would."""
import importlib.util
import os

import pytest

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_train_tokens():
    spec = importlib.util.spec_from_file_location("train_tokens", os.path.join(ROOT, "examples", "train_tokens.py"))
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    losses, drift = example.main(steps=40, verbose=False)
    assert losses[-1] < losses[0] - 2.0                  # of about log(4096) = 8.3 at first
    assert abs(losses[20] - losses[19]) < 1.0            # the step with a server down is like its neighbours
    assert drift < 1e-5                                  # entries of about 1: a few roundings of 2^-24 in each of 40 steps
