"""Pages that several sequences of a cache hold are read by all of them and written by none, on the CPU with the library's calls done by the oracle."""
import pytest

from paper_2402_02320_amd import spin
from test_cache_pages import Model, calls_of_the_oracle  # noqa: F401 - the calls' fixture


@pytest.fixture
def written(calls_of_the_oracle, monkeypatch):  # noqa: F811
    """Pages that compactions write, a list a call: rows context[b] + j of every kept row."""
    calls, compact = [], spin.cache_compact

    def watched(pools, table, context, kept, count):
        tokens = pools[0].shape[3]
        calls.append([int(table[b, (int(context[b]) + j) // tokens]) for b in range(table.shape[0]) for j in range(int(count[b]))])
        return compact(pools, table, context, kept, count)
    monkeypatch.setattr(spin, "cache_compact", watched)
    return calls


def shared(m):
    return {p for p, refs in enumerate(m.cache._refs) if refs > 1}


def test_rows_that_stay_are_not_written(written):
    m = Model(12)
    a, b = m.add(), m.add()
    m.append([a, b], [12, 12])
    c = m.fork(a)
    m.keep([a, b], 4, [[0, 1], [1, 3]])                       # a's stay, on a page that c has as well
    assert len(written) == 1 and not set(written[0]) & shared(m)
    m.check()
    m.keep([c], 4, [[0, 1, 2]])
    assert len(written) == 1                                  # nothing moves, nothing is called
    m.check()


def test_rows_before_the_first_that_moves_are_not_written(written):
    m = Model(12)
    a = m.add()
    m.append([a], [20])
    b = m.fork(a)
    before = shared(m)
    m.keep([a], 8, [[0, 1, 2, 3, 4, 6, 7]])                   # rows 12 to 16 stay, 18 and 19 move to 17 and 18 on a page of its own
    assert written == [[m.cache._pages[a][1]] * 2] and not set(written[0]) & shared(m) and shared(m) < before
    m.check()
    m.keep([b], 8, [[0, 1, 2, 3, 7]])
    m.check()
