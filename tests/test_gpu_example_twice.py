"""The small language model of examples/train_small_lm.py learns the same way twice, up to
the sums that torch's scatter leaves unordered."""
import importlib.util
import os

import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_small_lm_learns_the_same_way_twice():
    spec = importlib.util.spec_from_file_location(
        "train_small_lm", os.path.join(ROOT, "examples", "train_small_lm.py"))
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    first, second = example.train(rounds=4), example.train(rounds=4)
    # Other orders of a sum move gradients by some 1e-6 of their size, and turn the sign of
    # as small a share of the entries by the step of a round; the loss feels either by less
    # than a thousandth.
    for a, b in zip(first, second):
        assert abs(a - b) <= 1e-3 * a
