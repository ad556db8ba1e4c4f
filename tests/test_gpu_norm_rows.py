"""Layer norm, forward and backward, where a row belongs to four waves, and its gradient where a wave or workgroup has several rows and the last group fewer: word for word against
the numpy oracle.  tests/test_norm_rows.py checks on the CPU that each case is still what it says."""
import pytest
import torch

from oracle import linear as lin
import test_gpu_layernorm as norm
from test_gpu_generation import BITS, RINGS
from test_gpu_linattn import all_same, on

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
# name: (n, rows, dim, iterations), (waves and words a thread of a row, rows of a wave or workgroup), whether a kernel of their own makes the sums of columns (64-bit, 32-bit words)
SEVERAL_ROWS = {
    "a_wave_two": ((2, 4099, 40, 0), (1, 4, 2), (False, False)),
    "a_wave_three": ((3, 8197, 24, 0), (1, 4, 3), (False, False)),
    "a_wave_six": ((6, 4100, 255, 0), (1, 4, 2), (True, False)),
    "a_wave_seven": ((7, 4099, 40, 0), (1, 4, 2), (True, False)),
    "four_waves_three": ((3, 1029, 300, 0), (4, 4, 2), (False, False)),
    "four_waves_two": ((2, 2053, 260, 0), (4, 4, 3), (False, False)),
    "four_waves_six": ((6, 1029, 300, 0), (4, 4, 2), (True, False)),
    "four_waves_eight": ((8, 1027, 257, 0), (4, 4, 2), (True, False)),
    "sixteen_two_words": ((3, 515, 1030, 0), (16, 2, 3), (False, False)),
    "sixteen_two_words_eight": ((8, 259, 1025, 0), (16, 2, 2), (True, False)),
    "sixteen_four_words": ((2, 515, 2049, 0), (16, 4, 3), (False, False)),
    "sixteen_four_words_four": ((4, 259, 2049, 0), (16, 4, 2), (True, False)),
    "sixteen_eight_words": ((2, 301, 4100, 0), (16, 8, 2), (True, True)),
}
CASES = dict({"four_waves_" + k: v for k, v in FOUR_WAVES.items()}, **{"rows_" + k: v[0] for k, v in SEVERAL_ROWS.items()})


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


@BITS
def test_one_workspace_for_batches_of_all_sizes(bits):
    ring = RINGS[bits][0]
    ws = torch.full((ring.layernorm_grad_workspace_bytes(3, 1029, 300),), 0x5A, dtype=torch.uint8, device="cuda")
    for rows in (1029, 1024, 300, 256, 1, 1023):
        norm.CASES = {"batch": (3, rows, 300, 0)}
        args, more = norm.backward("batch", bits)
        assert all_same(ring.layernorm_grad(*on(args), *more, workspace=ws), lin.layernorm_grad(*args, *more)), rows
