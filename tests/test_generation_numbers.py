"""Numbers past 32 bits in the cache, attention and bias calls: the library takes ints, and ctypes would hand on their low halves.  On the CPU."""
import pytest
import torch

from paper_2402_02320_amd import spin
from test_generation_arguments import GOOD, record  # noqa: F401 - the library in whose place calls are written down

PAST = [2 ** 32, 2 ** 32 + 9, 2 ** 31, -2 ** 31 - 1, -2 ** 32 + 5]


@pytest.mark.parametrize("value", PAST)
@pytest.mark.parametrize("name,key", [("cache_scores", "f"), ("cache_values", "f"), ("relbias_trunc", "f"), ("relbias_trunc", "first"), ("relbias_grad", "first")])
def test_keywords(record, name, key, value):  # noqa: F811
    args, kw = GOOD[name]
    for ring in (spin, spin.ring32):
        with pytest.raises(spin.SpinError):
            getattr(ring, name)(*args, **{**kw, key: value})
    assert not record.launched


@pytest.mark.parametrize("value", PAST)
def test_buckets(record, value):  # noqa: F811
    (dS, lut, _), kw = GOOD["relbias_grad"]
    for ring in (spin, spin.ring32):
        with pytest.raises(spin.SpinError):
            ring.relbias_grad(dS, lut, value, out=torch.zeros(2, 6, 32, dtype=torch.int64).expand(2, 6, 32), **kw)
    assert not record.launched


def test_lengths_of_a_tensor(record):  # noqa: F811
    """As many keys as do not fit an int (of one word, expanded)."""
    x = torch.zeros(1, 1, 1, 1, 1, dtype=torch.int64).expand(1, 1, 1, 1, 2 ** 32 + 5)
    bias, lut = torch.zeros(1, 1, 4, dtype=torch.int64), torch.zeros(21, dtype=torch.int32)
    for call in (lambda: spin.relbias_trunc(x, bias, lut, out=x), lambda: spin.relbias_grad(x, lut, 4)):
        with pytest.raises(spin.SpinError):
            call()
    pool, table, one = torch.zeros(2, 1, 1, 16, 8, dtype=torch.int64), torch.zeros(1, 1, dtype=torch.int32), torch.zeros(1, dtype=torch.int32)
    Q = torch.zeros(1, 1, 1, 1, 8, dtype=torch.int64)
    for call in (lambda: spin.cache_scores(pool, table, one, Q, Q, x, out=x), lambda: spin.cache_values(pool, table, one, x, x, Q),
                 lambda: spin.cache_values_workspace_bytes(pool, table, 1, 1, 2 ** 32 + 5)):
        with pytest.raises(spin.SpinError):
            call()
    assert not record.launched
