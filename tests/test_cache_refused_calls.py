"""A call that the library refuses, or that fails on the way, leaves the pages of a cache as they were.  On the CPU, where the library refuses every tensor."""
import copy

import pytest
import torch

from paper_2402_02320_amd import spin
from paper_2402_02320_amd.cache import ShareCache
from test_cache_pages import DIM, HEADS, N, Model, calls_of_the_oracle  # noqa: F401 - the calls' fixture


def state(c):
    return copy.deepcopy((c._free, c._refs, c._pages, c._length))


def test_append_that_the_library_refuses(monkeypatch):
    monkeypatch.setattr(spin, "cache_append", spin._Word(64).cache_append)     # the library's own in place of the oracle's
    c = ShareCache(N, 6, HEADS, DIM, 16, device="cpu")
    a = c.add()
    before = state(c)
    x = torch.zeros(N, 1, HEADS, 20, DIM, dtype=torch.int64)
    with pytest.raises(spin.SpinError):
        c.append([a], (x, x), (x, x))                         # not on the GPU
    assert state(c) == before


@pytest.mark.parametrize("call", ["cache_append", "cache_copy"])
def test_append_that_fails_on_shared_pages(calls_of_the_oracle, monkeypatch, call):  # noqa: F811
    m = Model(8)
    a = m.add()
    m.append([a], [20])
    b = m.fork(a)
    before, rows = state(m.cache), {s: list(r) for s, r in m.rows.items()}

    def refuse(*args, **kw):
        raise spin.SpinError("refused")
    with monkeypatch.context() as refused:
        refused.setattr(spin, call, refuse)
        with pytest.raises(spin.SpinError, match="refused"):
            m.append([a, b], [30, 3])
    assert state(m.cache) == before and m.rows == rows
    m.check()
    m.append([a, b], [30, 3])
    m.check()


@pytest.mark.parametrize("call", ["cache_compact", "cache_copy"])
def test_keep_that_fails_on_shared_pages(calls_of_the_oracle, monkeypatch, call):  # noqa: F811
    m = Model(8)
    a = m.add()
    m.append([a], [20])
    m.fork(a)
    before = state(m.cache)

    def refuse(*args, **kw):
        raise spin.SpinError("refused")
    with monkeypatch.context() as refused:
        refused.setattr(spin, call, refuse)
        with pytest.raises(spin.SpinError, match="refused"):
            m.keep([a], 6, [[1, 5]])
    assert state(m.cache) == before
    m.check()
    m.keep([a], 6, [[1, 5]])
    m.check()
