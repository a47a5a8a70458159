"""The example of a training step: it learns, with the layers, their kept activations and the round together."""
import importlib.util
import os

import pytest
import torch

pytestmark = pytest.mark.gpu
PATH = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "train_residual.py")


@pytest.fixture(scope="module")
def example():
    spec = importlib.util.spec_from_file_location("train_residual", PATH)
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


def test_example_learns(example):
    """Ten equally likely classes: the loss starts near log 10 = 2.3 or above it, and ten fixed patterns are soon told apart."""
    losses, raw, sent = example.train(steps=40, workers=2)
    assert losses[0] > 1.5 and sum(losses[-5:]) / 5 < 0.5 * losses[0], losses
    assert sent < raw / 4


def test_example_repeats(example):
    """Sums have a fixed order: the same seed gives the same losses, bit for bit."""
    first, second = (example.train(steps=3, workers=2, seed=5)[0] for _ in range(2))
    assert first == second
