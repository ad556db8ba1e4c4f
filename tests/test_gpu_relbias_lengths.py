"""Lengths of every kind in the bias calls: below zero, near the ends of an int32, past the keys."""
import numpy as np
import pytest

from oracle import generation as gen
from test_gpu_generation import BITS, RINGS, dev, ints, same, tuple_of, uniform

pytestmark = pytest.mark.gpu

LOW, HIGH = -2 ** 31, 2 ** 31 - 1


@BITS
@pytest.mark.parametrize("Q,K", [(4, 4), (33, 300), (140, 9)])
@pytest.mark.parametrize("first,causal", [(0, False), (0, True), (60, True), (-3, False)])
def test_lengths_of_every_kind(bits, Q, K, first, causal):
    ring = RINGS[bits][0]
    rng = np.random.default_rng(Q + K + first)
    lengths = [LOW, LOW + 1, LOW + K, -1, 0, 1, K - 1, K, HIGH, LOW + 2]     # of the last matrix none is there either
    n, batch, heads, buckets = 2, len(lengths), 2, 16
    lut = rng.integers(0, buckets, size=2 * 20 + 1).astype(np.int32)
    x, table = uniform(rng, bits, n, batch, heads, Q, K), uniform(rng, bits, n, heads, buckets)
    kw = dict(first=first, causal=causal)
    got = ring.relbias_grad(dev(x), ints(lut), buckets, lengths=ints(lengths), **kw)
    assert same(got, gen.relbias_grad(x, lut, buckets, lengths=lengths, **kw))
    tup = tuple_of(rng, bits, x.shape)
    got = ring.relbias_trunc(dev(x), dev(table), ints(lut), f=9, tuple_=[dev(t) for t in tup], lengths=ints(lengths), masked=-99, **kw)
    assert same(got, gen.relbias_trunc(x, table, lut, 9, tup, lengths=lengths, masked=(1 << bits) - 99, **kw))
