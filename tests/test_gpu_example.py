"""The small language model of examples/train_small_lm.py learns its chain, and
learns it the same way twice up to the sums that torch's scatter leaves unordered."""
import importlib.util
import math
import os

import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_small_lm_learns():
    spec = importlib.util.spec_from_file_location(
        "train_small_lm", os.path.join(ROOT, "examples", "train_small_lm.py"))
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    losses = example.train(rounds=60)
    assert all(math.isfinite(v) for v in losses)
    # It starts at a uniform guess and ends far below.
    assert abs(losses[0] - math.log(example.VOCAB)) < 0.5
    assert losses[-1] < 0.7 * losses[0], losses[::10]
