"""The example that runs the 8-bit products, their gradients, the sparse exchange and the orthogonalised step together."""
import importlib.util
import os

import pytest

pytestmark = pytest.mark.gpu


def _example():
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "matrix_step.py")
    spec = importlib.util.spec_from_file_location("matrix_step", path)
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


@pytest.mark.parametrize("width, workers", [(200, 3), (75, 1)])
def test_the_example_learns(width, workers):
    losses = _example().train(width=width, tokens=300, workers=workers, steps=60, compression=20)
    # two networks that have nothing in common: the loss is about twice the answers' own variance at first
    assert losses[0] > 0.5
    assert sum(losses[-5:]) / 5 < 0.5 * losses[0]


def test_the_same_seed_takes_the_same_steps():
    train = _example().train
    assert train(width=96, tokens=64, workers=2, steps=6, seed=3) == train(width=96, tokens=64, workers=2, steps=6, seed=3)
