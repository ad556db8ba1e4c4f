"""Which page of a paged cache holds what: sequences that grow, fork, are cut back to an accepted draft and end, over the pools that spin.cache_append,
cache_copy, cache_compact, cache_scores and cache_values work on.

All bookkeeping is on the host; only the tables, lengths and page lists that the kernels read go to the device, with each call, by copies that the host waits for: none of these calls
can be captured into a graph.  Pages are handed on as soon as nothing refers to them,
so all calls on one cache belong on one stream (or are ordered otherwise)."""
import torch

from . import spin


_MOST_PAIRS = 65535                        # of one call of cache_copy


class ShareCache:
    """n parties, pages of page_tokens positions, `heads` cached heads of `dim` elements; bits: the ring's."""

    def __init__(self, n, pages, heads, dim, page_tokens=64, bits=64, device="cuda"):
        self.ring = {64: spin, 32: spin.ring32}[bits]
        shape = (n + 1, pages, heads, page_tokens, dim)
        self.pools = tuple(torch.empty(shape, dtype=torch.int64 if bits == 64 else torch.int32, device=device) for _ in range(2))
        self.page_tokens, self.device = page_tokens, device
        self._free = list(range(pages - 1, -1, -1))
        self._refs = [0] * pages
        self._pages, self._length, self._next = {}, {}, 0

    # ---- sequences ------------------------------------------------------------------------------------------------
    def add(self):
        """A new, empty sequence."""
        s, self._next = self._next, self._next + 1
        self._pages[s], self._length[s] = [], 0
        return s

    def fork(self, s):
        """A sequence with the same rows.  Nothing is copied until one of the two writes to a page that both have."""
        t = self.add()
        self._pages[t], self._length[t] = list(self._pages[s]), self._length[s]
        for p in self._pages[s]:
            self._refs[p] += 1
        return t

    def free(self, s):
        self._drop(self._pages.pop(s))
        del self._length[s]

    def length(self, s):
        return self._length[s]

    def pages_left(self):
        return len(self._free)

    def _drop(self, pages):
        for p in pages:
            self._refs[p] -= 1
            if not self._refs[p]:
                self._free.append(p)

    def _copy(self, pairs):
        """Copies pages (from, to), in as many calls as it takes: no page is written twice, or read and written."""
        for k in range(0, len(pairs), _MOST_PAIRS):
            src, dst = zip(*pairs[k:k + _MOST_PAIRS])
            self.ring.cache_copy(self.pools, self._ints(src), self._ints(dst))

    def _write(self, wanted, call):
        """Makes the pages of positions first to last - 1 of every (sequence, first, last) its own, new ones or copies of shared ones, and makes the call that writes
        to them.  All of it, or an error, and every sequence has the pages that it had."""
        t, plan = self.page_tokens, []
        refs = dict()
        for s, first, last in wanted:
            for k in range(first // t, -(-last // t)):
                p = self._pages[s][k] if k < len(self._pages[s]) else None
                if p is not None:
                    refs.setdefault(p, self._refs[p])
                    if refs[p] == 1:
                        continue
                    refs[p] -= 1
                plan.append((s, k, p))
        if len(plan) > len(self._free):
            raise spin.SpinError("the cache is out of pages: %d more are needed, %d are left" % (len(plan), len(self._free)))
        taken = []                                         # (sequence, which of its pages, the page before or None, its own)
        for s, k, p in plan:
            q = self._free.pop()
            self._refs[q] = 1
            taken.append((s, k, p, q))
            if p is None:
                assert k == len(self._pages[s])
                self._pages[s].append(q)
            else:
                self._refs[p] -= 1
                self._pages[s][k] = q
        filled = [(p, q) for s, k, p, q in taken if p is not None and k * t < self._length[s]]         # something is in it
        try:
            if filled:
                self._copy(filled)
            call()
        except BaseException:
            for s, k, p, q in reversed(taken):
                self._refs[q] = 0
                self._free.append(q)
                if p is None:
                    self._pages[s].pop()
                else:
                    self._refs[p] += 1
                    self._pages[s][k] = p
            raise

    # ---- what the kernels read ------------------------------------------------------------------------------------
    def _ints(self, v):
        return torch.tensor(v, dtype=torch.int32, device=self.device)

    def table(self, sequences):
        most = max(1, max(len(self._pages[s]) for s in sequences))
        return self._ints([self._pages[s] + [-1] * (most - len(self._pages[s])) for s in sequences])

    def context(self, sequences, nodes=0):
        """Lengths without the last `nodes` rows, the tokens that are being attended from."""
        return self._ints([self._length[s] - nodes for s in sequences])

    # ---- rows -----------------------------------------------------------------------------------------------------
    def append(self, sequences, x, b, counts=None):
        """Opens the rows x = (keys, values) against their masks b, [n, len(sequences), heads, rows, dim] each, and puts the first counts[k] (all of
        them by default) behind sequence k's."""
        if len(set(sequences)) < len(sequences):
            raise spin.SpinError("a sequence is appended to twice")
        rows = x[0].shape[3]
        counts = [rows] * len(sequences) if counts is None else list(counts)
        if len(counts) != len(sequences) or any(not 0 <= c <= rows for c in counts):
            raise spin.SpinError("counts: one for every sequence, none over the number of rows")
        self._write([(s, self._length[s], self._length[s] + c) for s, c in zip(sequences, counts) if c],
                    lambda: self.ring.cache_append(self.pools, self.table(sequences), self.context(sequences), x, b, count=self._ints(counts)))
        for s, c in zip(sequences, counts):
            self._length[s] += c

    def keep(self, sequences, nodes, kept):
        """Of the last `nodes` rows of every sequence, a draft, keeps those listed in kept[k], ascending: they move together, and the pages behind them are free again."""
        if len(set(sequences)) < len(sequences) or len(kept) != len(sequences):
            raise spin.SpinError("a list of kept rows for every sequence, once")
        for s, k in zip(sequences, kept):
            if not 0 <= nodes <= self._length[s] or any(not 0 <= a < nodes for a in k) or any(a >= b for a, b in zip(k, k[1:])):
                raise spin.SpinError("kept rows are ascending indices into the draft")
        moved = []                                         # (sequence, position of the first row that moves, the rows from there on)
        for s, k in zip(sequences, kept):
            j = next((j for j, a in enumerate(k) if a != j), None)
            if j is not None:
                moved.append((s, self._length[s] - nodes + j, [a - j for a in list(k)[j:]]))
        if moved:                                          # nothing else is handed over: what stays may be on pages that others have too
            self._write([(s, first, first + len(k)) for s, first, k in moved],
                        lambda: self.ring.cache_compact(self.pools, self.table([s for s, _, _ in moved]), self._ints([first for _, first, _ in moved]),
                                                        self._ints([k + [0] * (nodes - len(k)) for _, _, k in moved]), self._ints([len(k) for _, _, k in moved])))
        for s, k in zip(sequences, kept):
            self._length[s] += len(k) - nodes
            used = -(-self._length[s] // self.page_tokens)
            self._drop(self._pages[s][used:])
            del self._pages[s][used:]

    def compact(self):
        """Moves pages to the front of the pools; how many are in use, which are then the first ones."""
        used = {p for p, r in enumerate(self._refs) if r}
        low = [p for p in range(len(used)) if p not in used]
        moved = dict(zip(sorted(p for p in used if p >= len(used)), low))
        if moved:
            self._copy(list(moved.items()))
            for pages in self._pages.values():
                pages[:] = [moved.get(p, p) for p in pages]
            for p, q in moved.items():
                self._refs[q], self._refs[p] = self._refs[p], 0
            self._free = [p for p in range(len(self._refs) - 1, -1, -1) if not self._refs[p]]
        return len(used)
