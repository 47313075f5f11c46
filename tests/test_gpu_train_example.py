"""The training example runs end to end and learns, compressed and not."""
import importlib.util
import os

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def example():
    spec = importlib.util.spec_from_file_location("train_compressed", os.path.join(ROOT, "examples", "train_compressed.py"))
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


@pytest.mark.parametrize("compressed", [True, False])
def test_training_learns(example, compressed):
    losses, share = example.train(steps=60, compressed=compressed, tell=lambda *_: None)
    assert all(l == l for l in losses)
    assert sum(losses[-5:]) < 0.5 * sum(losses[:5])
    assert share < 0.6 if compressed else share == 1.0


def test_training_repeats_bit_for_bit(example):
    a, _ = example.train(steps=12, tell=lambda *_: None)
    b, _ = example.train(steps=12, tell=lambda *_: None)
    assert a == b
