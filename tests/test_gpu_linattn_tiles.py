"""Linear attention on so many chunks that its products are made by tiles of 64 (64-bit words): one to eight parties, odd widths, cut, empty and overlong
sequences, whole and half tiles of a chunk.  Word for word against the numpy oracle; each case is checked to be of that many tiles, so that another choice of
tiles cannot take them out of the tests unseen."""
import os
import re

import pytest

from paper_2402_02320_amd import build
import test_gpu_linattn as small
from test_gpu_linattn import Case, all_same, both, same

pytestmark = pytest.mark.gpu

# n, batch, heads, tokens, rows, columns, chunk, lengths, f, g
CASES = {
    "one_party": (1, 4, 8, 520, 64, 64, 64, (520, 449, 0, 64), 16, 12),
    "two_odd": (2, 2, 4, 1000, 72, 136, 128, (1000, 577), 16, 12),
    "three_narrow_keys": (3, 3, 8, 700, 40, 200, 64, (700, -1, 65), 16, 12),
    "three_no_decay": (3, 1, 16, 512, 96, 72, 128, None, 16, None),
    "four": (4, 2, 8, 500, 72, 104, 128, (500, 129), 16, 12),
    "five_wide_keys": (5, 2, 8, 500, 256, 72, 128, (900, 320), 16, 12),
    "eight": (8, 2, 8, 500, 72, 72, 128, (400, 193), 9, 6),
}
NAMES = pytest.mark.parametrize("name", sorted(CASES))


@pytest.fixture(autouse=True)
def cases(monkeypatch):
    monkeypatch.setattr(small, "CASES", CASES)


def by_64(c, rows, columns):
    with open(os.path.join(build.CSRC, "linattn.hip")) as source:
        wanted = int(re.search(r"kWantedTiles = (\d+);", source.read()).group(1))
    return min(rows, columns) > 32 and c.batch * c.heads * c.chunks * -(-rows // 64) * -(-columns // 64) >= wanted


@NAMES
def test_scores(name):
    c = Case(name, 64)
    assert by_64(c, c.chunk, c.chunk)
    C, t = c.dealt(c.chunks, c.chunk, c.chunk)
    want, call, ops = both(c, "scores", c.factor(c.tokens, c.dk), c.factor(c.tokens, c.dk), C, t)
    assert same(call(), want)
    assert same(call(out=ops[3][2]), want)                    # in place of a tuple's r_msb


@pytest.mark.parametrize("reverse", [False, True])
@NAMES
def test_states(name, reverse):
    c = Case(name, 64)
    assert by_64(c, c.dk, c.dv)
    C, t = c.dealt(c.chunks, c.dk, c.dv)
    want, call, _ = both(c, "states", c.factor(c.tokens, c.dk), c.factor(c.tokens, c.dv), C, t, reverse=reverse, first=c.u(c.dk, c.dv), chunk=c.chunk)
    assert all_same(call(), want)


@pytest.mark.parametrize("reverse,transposed", [(False, False), (False, True), (True, False), (True, True)])
@NAMES
def test_outputs(name, reverse, transposed):
    c = Case(name, 64)
    assert by_64(c, c.chunk, c.dv)
    C, t = c.dealt(c.tokens, c.dv)
    state = (c.dv, c.dk) if transposed else (c.dk, c.dv)
    want, call, ops = both(c, "outputs", c.factor(c.chunks, c.chunk, c.chunk), c.factor(c.tokens, c.dv), c.factor(c.tokens, c.dk), c.factor(c.chunks, *state), C, t,
                           reverse=reverse, transposed=transposed)
    assert same(call(), want)
    assert same(call(out=ops[4]), want)                       # in place of C
