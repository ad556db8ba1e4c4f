"""More pages than one copy call takes, on the CPU with the copies written down."""
import pytest
import torch

from paper_2402_02320_amd import spin
from paper_2402_02320_amd.cache import ShareCache

MOST = 65535                               # pairs of one call: spin_cache_copy refuses more


@pytest.fixture
def copies(monkeypatch):
    made = []

    def copy(pools, src, dst):
        if src.numel() > MOST:
            raise spin.SpinError("too many")
        made.append(list(zip(src.tolist(), dst.tolist())))
    monkeypatch.setattr(spin, "cache_copy", copy)
    monkeypatch.setattr(spin, "cache_append", lambda *a, **kw: None)
    return made


def small(pages):
    return ShareCache(1, pages, 1, 8, 16, device="cpu")       # its pools are never touched


def filled(c, count, rows):
    """`count` sequences of `rows` rows each."""
    some = [c.add() for _ in range(count)]
    x = torch.zeros(1, 1, 1, rows, 8, dtype=torch.int64).expand(1, count, 1, rows, 8)
    c.append(some, (x, x), (x, x))
    return some


def test_forks_of_more_sequences_than_a_call_copies(copies):
    count = MOST + 3
    c = small(2 * count)
    some = filled(c, count, 1)
    for s in some:
        c.fork(s)
    before = {s: c._pages[s][0] for s in some}
    x = torch.zeros(1, 1, 1, 1, 8, dtype=torch.int64).expand(1, count, 1, 1, 8)
    c.append(some, (x, x), (x, x))
    assert [len(m) for m in copies] == [MOST, 3]
    assert {p: q for m in copies for p, q in m} == {before[s]: c._pages[s][0] for s in some}


def test_compaction_of_more_pages_than_a_call_copies(copies):
    count = MOST + 3
    c = small(2 * count)
    first, rest = filled(c, count, 1), filled(c, count, 1)
    for s in first:
        c.free(s)
    before = {s: c._pages[s][0] for s in rest}
    assert c.compact() == count
    assert [len(m) for m in copies] == [MOST, 3]
    moved = {p: q for m in copies for p, q in m}
    assert all(c._pages[s][0] == moved[before[s]] < count for s in rest)
