"""The host side of the paged cache: pages of growing, forked, cut and freed sequences, on the CPU with the library's three calls done by the oracle.  Every sequence has to
read back what was appended to it, whatever the others did."""
import numpy as np
import pytest
import torch

from oracle import generation as gen
from paper_2402_02320_amd import spin
from paper_2402_02320_amd.cache import ShareCache

N, HEADS, DIM = 2, 1, 8


@pytest.fixture(autouse=True)
def calls_of_the_oracle(monkeypatch):
    def put(pools, new):
        for p, q in zip(pools, new):
            p.copy_(torch.from_numpy(q.view(np.int64)))

    def words(t):
        return t.numpy().view(np.uint64)
    monkeypatch.setattr(spin, "cache_append", lambda pools, table, start, x, b, count=None: put(
        pools, [gen.append(words(p), table.numpy(), start.numpy(), count.numpy(), words(u), words(v)) for p, u, v in zip(pools, x, b)]))

    def copy(pools, src, dst):
        assert len(set(dst.tolist())) == len(dst) and not set(src.tolist()) & set(dst.tolist())
        put(pools, [gen.copy(words(p), src.tolist(), dst.tolist()) for p in pools])
    monkeypatch.setattr(spin, "cache_copy", copy)
    monkeypatch.setattr(spin, "cache_compact", lambda pools, table, context, kept, count: put(
        pools, [gen.compact(words(p), table.numpy(), context.numpy(), kept.numpy(), count.numpy()) for p in pools]))


class Model:
    """A cache, and beside it what every sequence should hold: rows are told apart by their value."""

    def __init__(self, pages, tokens=16):
        self.cache, self.rows, self.stamp = ShareCache(N, pages, HEADS, DIM, tokens, device="cpu"), {}, 1
        for p in self.cache.pools:
            p.zero_()

    def add(self):
        s = self.cache.add()
        self.rows[s] = []
        return s

    def fork(self, s):
        t = self.cache.fork(s)
        self.rows[t] = list(self.rows[s])
        return t

    def free(self, s):
        self.cache.free(s)
        del self.rows[s]

    def append(self, sequences, counts):
        rows = max(counts)
        x = torch.zeros(N, len(sequences), HEADS, max(rows, 1), DIM, dtype=torch.int64)
        values = [list(range(self.stamp + 100 * k, self.stamp + 100 * k + rows)) for k in range(len(sequences))]
        self.stamp += 100 * len(sequences)
        for k, v in enumerate(values):
            for j, w in enumerate(v):
                x[0, k, :, j] = w
        b = torch.randint(-2 ** 62, 2 ** 62, x.shape)
        self.cache.append(sequences, (x, -x), (b, b), counts)
        for s, v, c in zip(sequences, values, counts):
            self.rows[s] += v[:c]

    def keep(self, sequences, nodes, kept):
        self.cache.keep(sequences, nodes, kept)
        for s, k in zip(sequences, kept):
            draft = self.rows[s][len(self.rows[s]) - nodes:]
            self.rows[s][len(self.rows[s]) - nodes:] = [draft[a] for a in k]

    def check(self):
        for s, want in self.rows.items():
            assert self.cache.length(s) == len(want) and len(self.cache._pages[s]) == -(-len(want) // self.cache.page_tokens)
            if not want:
                continue
            table = self.cache.table([s]).numpy()
            for sign, pool in zip((1, -1), self.cache.pools):
                got = gen.cached_rows(pool.numpy().view(np.uint64), table, 0, 0, len(want))[1:].sum(0, dtype=np.uint64).view(np.int64)
                assert got[:, 0].tolist() == [sign * w for w in want]
        held = [p for pages in self.cache._pages.values() for p in pages]
        assert [held.count(p) for p in range(len(self.cache._refs))] == self.cache._refs
        assert sorted(self.cache._free + sorted(set(held))) == list(range(len(self.cache._refs)))


def test_fork_copies_when_written():
    m = Model(8)
    a = m.add()
    m.append([a], [20])
    b = m.fork(a)
    assert m.cache.pages_left() == 6
    m.append([a, b], [3, 2])                                  # one of the two copies the half-filled page, the other keeps it
    assert m.cache.pages_left() == 5
    m.check()
    c = m.fork(b)
    m.keep([b], 4, [[1, 3]])                                  # rows that move on a shared page
    m.check()
    for s in (a, b, c):
        m.free(s)
    assert m.cache.pages_left() == 8 and not any(m.cache._refs)


def test_out_of_pages_changes_nothing():
    m = Model(3)
    a, b = m.add(), m.add()
    m.append([a], [40])
    with pytest.raises(spin.SpinError, match="out of pages"):
        m.append([a, b], [2, 1])
    m.check()
    m.keep([a], 9, [[]])
    m.append([b], [16])
    m.check()


def test_refusals():
    m = Model(4)
    a = m.add()
    m.append([a], [5])
    for bad in (lambda: m.cache.keep([a], 6, [[0]]), lambda: m.cache.keep([a], 3, [[1, 1]]), lambda: m.cache.keep([a], 3, [[2, 1]]), lambda: m.cache.keep([a], 3, [[3]]),
                lambda: m.cache.keep([a], 3, []), lambda: m.append([a, a], [1, 1]), lambda: m.cache.append([a], (torch.zeros(2, 1, 1, 2, 8),) * 2, None, [3])):
        with pytest.raises(spin.SpinError):
            bad()
    m.check()


def test_compaction_moves_to_the_front():
    m = Model(10)
    s = [m.add() for _ in range(4)]
    m.append(s, [33, 16, 17, 1])
    t = m.fork(s[2])
    m.free(s[0])
    assert m.cache.compact() == 4
    assert all(p < 4 for pages in m.cache._pages.values() for p in pages)
    m.append([t], [20])
    m.check()


@pytest.mark.parametrize("seed", range(12))
def test_any_history(seed):
    rng = np.random.default_rng(seed)
    m = Model(24)
    for _ in range(60):
        live = list(m.rows)
        act = rng.integers(0, 7)
        if act == 0 or not live:
            m.add()
        elif act == 1 and len(live) < 6:
            m.fork(int(rng.choice(live)))
        elif act == 2 and len(live) > 2:
            m.free(int(rng.choice(live)))
        elif act == 3:
            m.cache.compact()
        else:
            some = [int(s) for s in rng.permutation(live)[:rng.integers(1, 4)]]
            try:
                if act == 4 and min(len(m.rows[s]) for s in some) >= 5:
                    m.keep(some, 5, [sorted(rng.permutation(5)[:rng.integers(0, 6)].tolist()) for _ in some])
                else:
                    m.append(some, [int(c) for c in rng.integers(0, 20, len(some))])
            except spin.SpinError:
                pass
        m.check()
