"""The example that trains and serves with the layers: it learns, with moments in 8 bits as with 32, and runs again the same."""
import importlib.util
import os

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def example():
    spec = importlib.util.spec_from_file_location("feed_forward", os.path.join(ROOT, "examples", "feed_forward.py"))
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


@pytest.mark.parametrize("bits", [8, 32])
def test_training_learns(example, bits):
    losses = example.train(120, bits=bits)
    assert losses[-1] < 0.5 * losses[0]
    assert losses == example.train(120, bits=bits)


def test_serving(example):
    norms, taken = example.serve()
    assert len(norms) == 8 and all(n > 0 for n in norms)
    assert all(0 <= a < b < 16 for a, b in taken)
    assert (norms, taken) == example.serve()
