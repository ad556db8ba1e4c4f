"""Linear attention of as many parties as the other tests leave out: tiles of 64 take masks three parties at a time, so that six parties have a last part that is whole, seven one of a
single party; the states of six go over the chunks two at a time; single tokens of four, five and seven.  Word for word against the numpy oracle."""
import pytest

import test_gpu_linattn as small
import test_gpu_linattn_tiles as tiles
from test_gpu_linattn import BITS

pytestmark = pytest.mark.gpu

# n, batch, heads, tokens, rows, columns, chunk, lengths, f, g
SMALL = {
    "six_odd": (6, 3, 2, 300, 40, 72, 128, (300, 129, 0), 16, 12),
    "six_one_chunk": (6, 1, 1, 33, 8, 256, 64, None, 9, 6),
    "six_three_chunks": (6, 2, 1, 96, 64, 16, 32, (96, 65), 16, None),
    "seven_odd": (7, 2, 1, 161, 136, 24, 32, (161, 64), 9, 6),
}
BY_64 = {
    "six": (6, 3, 8, 500, 72, 104, 128, (500, 129, 0), 16, 12),
    "six_short_chunks": (6, 2, 8, 1024, 40, 64, 64, (1024, 577), 9, 6),
    "seven": (7, 3, 8, 500, 104, 72, 128, (500, -3, 257), 16, 12),
    "seven_no_decay": (7, 1, 16, 512, 72, 136, 128, None, 9, None),
}
STEPS = {                                                     # n, batch, heads, rows, columns, active, f, g
    "four": (4, 3, 2, 72, 104, (1, 0, 1), 16, 12),
    "five": (5, 2, 3, 64, 64, None, 16, 12),
    "seven": (7, 2, 2, 40, 136, (0, 1), 9, 6),
}
ALL = SMALL | BY_64
BOTH_WAYS = pytest.mark.parametrize("reverse", [False, True])
TRANSPOSED = pytest.mark.parametrize("transposed", [False, True])


@pytest.fixture(autouse=True)
def cases(monkeypatch):
    monkeypatch.setattr(small, "CASES", ALL)
    monkeypatch.setattr(small, "STEPS", STEPS)


@BITS
@pytest.mark.parametrize("name", sorted(SMALL))
def test_scores(name, bits):
    small.test_scores(name, bits)


@BITS
@BOTH_WAYS
@pytest.mark.parametrize("name", sorted(SMALL))
def test_states(name, reverse, bits):
    small.test_states(name, reverse, bits)


@BITS
@BOTH_WAYS
@TRANSPOSED
@pytest.mark.parametrize("name", sorted(SMALL))
def test_outputs(name, transposed, reverse, bits):
    small.test_outputs(name, reverse, transposed, bits)


@pytest.mark.parametrize("name", sorted(BY_64))
def test_scores_by_64(name):
    tiles.test_scores(name)


@BOTH_WAYS
@pytest.mark.parametrize("name", sorted(BY_64))
def test_states_by_64(name, reverse):
    tiles.test_states(name, reverse)


@BOTH_WAYS
@TRANSPOSED
@pytest.mark.parametrize("name", sorted(BY_64))
def test_outputs_by_64(name, transposed, reverse):
    tiles.test_outputs(name, reverse, transposed)


@BITS
@pytest.mark.parametrize("name", sorted(STEPS))
def test_step(name, bits):
    small.test_step(name, bits)
