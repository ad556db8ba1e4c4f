"""Layer norm, forward and backward, where a row belongs to four waves: word for word against the numpy oracle.  tests/test_norm_rows.py checks on the CPU that each case is still what it says."""
import pytest

import test_gpu_layernorm as norm
from test_gpu_generation import BITS

pytestmark = pytest.mark.gpu

# name: n, rows, dim, iterations
FOUR_WAVES = {
    "one_party": (1, 258, 512, 2),
    "two_odd": (2, 300, 333, 3),
    "three_whole": (3, 257, 1024, 4),
    "four": (4, 270, 500, 2),
    "five_narrow": (5, 1100, 257, 2),
    "six": (6, 261, 640, 1),
    "seven": (7, 259, 1023, 1),
    "eight": (8, 260, 777, 1),
}
CASES = {"four_waves_" + k: v for k, v in FOUR_WAVES.items()}



@pytest.fixture(autouse=True)
def cases(monkeypatch):
    monkeypatch.setattr(norm, "CASES", CASES)


@BITS
@pytest.mark.parametrize("name", sorted(FOUR_WAVES))
def test_forward_by_four_waves(name, bits):
    norm.test_forward("four_waves_" + name, bits)


@BITS
@pytest.mark.parametrize("name", sorted(CASES))
def test_backward(name, bits):
    norm.test_backward(name, bits)
