"""examples/generate.py: cache, drafted attention, page moves and the bias's training run together, against float64."""
import importlib.util
import os

import pytest

pytestmark = pytest.mark.gpu
PATH = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "generate.py")


@pytest.fixture(scope="module")
def example():
    spec = importlib.util.spec_from_file_location("generate_example", PATH)
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


@pytest.mark.parametrize("n,heads,cached,dim", [(3, 8, 2, 64), (2, 4, 4, 40)])
def test_drafted_attention(example, n, heads, cached, dim):
    """Fixed point of 16 bits: encoding moves every factor by less than 2^-16, a sum of dim products of sizes about 0.3 and 5 at most by dim * 1.5 * 2^-16, softmax of scores
    off by d is off by at most 2 d relative to itself, and values up to 5 are weighted by weights that are encoded again over at most 100 rows."""
    worst, used = example.generate(n, heads, cached, dim)
    score = dim * 3 * 2.0 ** -16 + 2.0 ** -15
    assert worst <= 5 * 2 * score + 100 * 5 * 2.0 ** -16 + 2.0 ** -15
    assert 0 < used < 32


def test_the_bias_learns(example):
    """Every bucket of a head moves towards its hidden value (a positive step of at most one), so no distance grows by more than the roundings."""
    losses = example.train_bias()
    assert all(b <= a + 2.0 ** -14 for a, b in zip(losses, losses[1:])) and losses[-1] < losses[0]
