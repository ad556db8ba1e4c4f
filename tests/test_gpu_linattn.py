"""Linear attention with a decay on shares, word for word against the numpy oracle: both rings, one to eight parties, every chunk length, cut and empty
chunks, odd widths, gradients, single tokens, other streams, graphs, results in place of their operands."""
import numpy as np
import pytest
import torch

from oracle import linear as lin
from paper_2402_02320_amd import spin
from test_gpu_generation import BITS, RINGS, dev, ints, same, tuple_of, uniform

pytestmark = pytest.mark.gpu


def on(v):
    """Host arrays in tuples and lists, on the GPU."""
    return None if v is None else dev(v) if isinstance(v, np.ndarray) else type(v)(on(k) for k in v)


def all_same(got, want):
    return all(same(g, w) for g, w in zip(got, want)) and len(got) == len(want)


# name: n, batch, heads, tokens, rows (of keys), columns (of values), chunk, lengths, f, g (None: no decay)
CASES = {
    "one_token": (3, 1, 2, 1, 16, 24, 32, None, 16, 12),
    "one_party": (1, 1, 1, 5, 8, 8, 32, None, 3, 2),
    "one_chunk": (2, 1, 2, 64, 64, 64, 64, None, 16, 12),
    "cut_and_empty": (3, 4, 2, 100, 40, 72, 32, (100, 33, 0, 64), 16, 12),
    "negative_and_long": (2, 3, 1, 70, 16, 16, 64, (-5, 999, 1), 16, 12),
    "no_decay": (3, 2, 2, 150, 64, 32, 64, (150, 65), 16, None),
    "wide": (2, 1, 2, 130, 256, 200, 64, None, 16, 12),
    "chunk_128": (3, 2, 2, 300, 128, 128, 128, (300, 129), 16, 12),
    "chunk_128_odd": (2, 2, 3, 259, 72, 136, 128, (259, 200), 16, 12),
    "five_parties": (5, 2, 1, 97, 48, 80, 32, (97, 40), 16, 12),
    "eight_parties": (8, 1, 2, 129, 64, 64, 128, None, 9, 6),
    "four_parties_wide": (4, 1, 1, 66, 256, 256, 32, None, 9, 6),
    "seven_parties": (7, 1, 1, 33, 24, 8, 64, None, 9, 6),
}


class Case:
    def __init__(self, name, bits, seed=0):
        self.n, self.batch, self.heads, self.tokens, self.dk, self.dv, self.chunk, lengths, f, g = CASES[name]
        self.bits, self.rng = bits, np.random.default_rng(seed + sum(map(ord, name)))
        self.ring = RINGS[bits][0]
        f, g = (f, g) if bits == 64 else (9, g and 6)
        self.host = dict(f=f, g=g or 0, lengths=None if lengths is None else np.array(lengths), decay=None)
        if g:
            self.host["decay"] = np.array([[round((1 - 2.0 ** -(2 + h)) ** j * 2 ** g) for j in range(self.chunk + 1)] for h in range(self.heads)], RINGS[bits][1])
            self.host["decay"][-1] = uniform(self.rng, bits, self.chunk + 1)                  # weights are any words
        self.device = dict(self.host, lengths=None if lengths is None else ints(lengths), decay=on(self.host["decay"]))
        self.chunks = -(-self.tokens // self.chunk)

    def u(self, *shape):
        return uniform(self.rng, self.bits, self.n, self.batch, self.heads, *shape)

    def factor(self, *shape):
        return self.u(*shape), self.u(*shape)

    def dealt(self, *shape):
        return self.u(*shape), [self.u(*shape) for _ in range(3)]


def both(c, name, *args, **more):
    """The oracle's result, and a call of the library's on the same operands."""
    ops = [on(a) if isinstance(a, (np.ndarray, tuple, list)) else a for a in args]
    kept = {k: on(v) if isinstance(v, np.ndarray) else v for k, v in more.items()}
    return getattr(lin, name)(*args, **more, **c.host), lambda **kw: getattr(c.ring, "linattn_" + name)(*ops, **kept, **c.device, **kw), ops


@BITS
@pytest.mark.parametrize("name", sorted(CASES))
def test_scores(name, bits):
    c = Case(name, bits)
    C, t = c.dealt(c.chunks, c.chunk, c.chunk)
    want, call, ops = both(c, "scores", c.factor(c.tokens, c.dk), c.factor(c.tokens, c.dk), C, t)
    assert same(call(), want)
    assert same(call(out=ops[2]), want)                       # in place of C


@BITS
@pytest.mark.parametrize("reverse", [False, True])
@pytest.mark.parametrize("name", sorted(CASES))
def test_states(name, reverse, bits):
    c = Case(name, bits)
    C, t = c.dealt(c.chunks, c.dk, c.dv)
    x, y, first = c.factor(c.tokens, c.dk), c.factor(c.tokens, c.dv), c.u(c.dk, c.dv)
    for start in (first, None):
        want, call, ops = both(c, "states", x, y, C, t, reverse=reverse, first=start, chunk=c.chunk)
        assert all_same(call(), want)
    need = c.ring.linattn_states_workspace_bytes(c.n, c.batch, c.heads, c.tokens, c.chunk, c.dk, c.dv)
    ws = torch.full((need + 512,), 0x5A, dtype=torch.uint8, device="cuda")
    assert all_same(call(workspace=ws[:need]), want) and bool((ws[need:] == 0x5A).all())
    last = torch.empty(first.shape, dtype=ops[2].dtype, device="cuda")
    assert all_same(call(out=(ops[2], last)), want)           # in place of C


@BITS
@pytest.mark.parametrize("reverse,transposed", [(False, False), (False, True), (True, False), (True, True)])
@pytest.mark.parametrize("name", sorted(CASES))
def test_outputs(name, reverse, transposed, bits):
    c = Case(name, bits)
    C, t = c.dealt(c.tokens, c.dv)
    state = (c.dv, c.dk) if transposed else (c.dk, c.dv)
    want, call, ops = both(c, "outputs", c.factor(c.chunks, c.chunk, c.chunk), c.factor(c.tokens, c.dv), c.factor(c.tokens, c.dk), c.factor(c.chunks, *state), C, t,
                           reverse=reverse, transposed=transposed)
    assert same(call(), want)
    assert same(call(out=ops[5][1]), want)                    # in place of a tuple's r_top


STEPS = {                                                     # n, batch, heads, rows, columns, active, f, g
    "token": (3, 1, 1, 64, 64, None, 16, 12),
    "idle": (3, 5, 2, 40, 72, (1, 0, 7, -1, 1), 16, 12),
    "smallest": (1, 1, 1, 8, 8, None, 3, None),
    "widest": (2, 2, 2, 256, 256, None, 16, 12),
    "tall": (2, 1, 3, 256, 8, None, 16, None),
    "flat": (2, 1, 3, 8, 200, None, 16, 12),
    "eight": (8, 2, 2, 128, 128, (1, 1), 9, 6),
    "six": (6, 1, 2, 96, 40, None, 9, 6),
    "many": (2, 33, 4, 64, 128, None, 16, 12),
}


@BITS
@pytest.mark.parametrize("name", sorted(STEPS))
def test_step(name, bits):
    n, batch, heads, rows, columns, active, f, g = STEPS[name]
    f, g = (f, g) if bits == 64 else (9, g and 6)
    rng = np.random.default_rng(sum(map(ord, name)))
    ring = RINGS[bits][0]

    def u(*shape):
        return uniform(rng, bits, n, batch, heads, *shape)
    decay = uniform(rng, bits, heads, 2) if g else None
    state = (rows, columns)
    args = (u(*state), (u(rows), u(rows)), (u(rows), u(rows)), (u(columns), u(columns)), u(*state), (u(*state), u(columns)),
            ([u(*state) for _ in range(3)], [u(columns) for _ in range(3)]))
    want = lin.step(*args, f, decay, g or 0, active)
    ops = on(args)
    more = dict(decay=on(decay), g=g or 0, active=None if active is None else ints(active))
    assert all_same(ring.linattn_step(*ops, f, **more), want)
    out = torch.empty_like(ops[5][1])
    assert all_same(ring.linattn_step(*ops, f, out=(out, ops[0]), **more), want) and same(ops[0], want[1])      # the state in its place
