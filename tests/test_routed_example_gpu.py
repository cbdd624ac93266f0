"""The example of a routed layer: it learns, and the potentials spread the tokens over the experts."""
import importlib.util
import os

import pytest

pytestmark = pytest.mark.gpu

PATH = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "routed_layer.py")


def test_example_learns_and_balances():
    spec = importlib.util.spec_from_file_location("routed_layer_example", PATH)
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    losses, spread = example.main(steps=30, say=None)
    assert losses[-1] < 0.7 * losses[0]
    _, free = example.main(steps=1, balanced=False, say=None)
    assert spread[0] < free[0]
    assert max(spread) < 1.6
