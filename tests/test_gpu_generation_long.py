"""Attention over caches so long that one workgroup has several turns of tokens (values) or several runs (scores): random words, pages in any order, contexts
that end inside a later turn or run.  Word for word against the formula in elementwise torch operations; each case says how many turns or runs it is for, so
that another choice of ranges cannot take them out of the tests unseen."""
import os
import re

import pytest
import torch

from paper_2402_02320_amd import build, spin
from test_gpu_generation import RINGS, ints

pytestmark = pytest.mark.gpu
TOKENS = 64                                # of a turn, and of a run


def words(bits, *shape):
    return torch.empty(shape, dtype=torch.int64 if bits == 64 else torch.int32, device="cuda").random_(-2 ** (bits - 1), 2 ** (bits - 1) - 1)


class Case:
    def __init__(self, seed, bits, n, batch, kv, share, nodes, dim, columns, tokens=32):
        torch.manual_seed(seed)
        self.bits, self.n, self.batch, self.kv, self.share, self.nodes, self.dim, self.columns, self.tokens = bits, n, batch, kv, share, nodes, dim, columns, tokens
        self.ring, self.heads = RINGS[bits][0], kv * share
        pages = 100
        self.pool = words(bits, n + 1, pages, kv, tokens, dim)
        self.table = torch.randint(0, pages, (batch, -(-columns // tokens)), device="cuda").int()      # shared pages are read by all
        self.table[0, 3], self.table[-1, 5] = -1, pages       # pages that are not there
        most = columns - nodes
        self.contexts = [most, most - 1, most - 70, most // 2 + 5, 200, 3 * TOKENS - 1, 0, -1][:batch] + [most - 37 * k for k in range(8, batch)]
        self.context = ints(self.contexts)
        bits_of = torch.randint(0, 1 << nodes, (batch, nodes), device="cuda")
        self.tree = bits_of | (1 << torch.arange(nodes, device="cuda"))
        self.depth = torch.randint(0, 5, (batch, nodes), device="cuda").int()
        at = torch.arange(columns, device="cuda") - self.context[:, None, None]
        there = self.table[:, torch.arange(columns, device="cuda") // tokens]
        self.seen = (at < 0) | ((at < nodes) & ((self.tree[:, :, None] >> at.clamp(0, nodes - 1)) & 1 > 0))
        self.seen &= (self.context[:, None, None] >= 0) & ((there >= 0) & (there < pages))[:, None]

    def rows(self, b):
        """[slots, kv, columns, dim] of a sequence; where no page is there, of some other."""
        got = self.pool[:, self.table[b].long().clamp(0, self.pool.shape[1] - 1)].transpose(1, 2)
        return got.reshape(self.n + 1, self.kv, -1, self.dim)[:, :, :self.columns]

    def products(self, x, A, C, transposed):
        """C + E . slot(1 + i) + A_i . slot(0), before truncation.  transposed: rows of scores, otherwise sums of values."""
        out = C.clone()
        E = (x - A).sum(0, dtype=x.dtype)
        axis = -1 if transposed else -2
        for b in range(self.batch):
            rows = self.rows(b)
            for h in range(self.heads):
                for m in range(self.nodes):
                    e, a = E[b, h, m], A[:, b, h, m]
                    of = rows[:, h // self.share]
                    e, a = (e[None, None, :], a[:, None, :]) if transposed else (e[None, :, None], a[:, :, None])
                    out[:, b, h, m] += (e * of[1:]).sum(axis, dtype=x.dtype) + (a * of[0]).sum(axis, dtype=x.dtype)
        return out

    def truncated(self, z, f, tup):
        return self.ring.trunc(z.reshape(self.n, -1), *[t.reshape(self.n, -1) for t in tup], f).view(z.shape) if f else z


# bits, n, batch, cached heads, query heads of each, nodes, dim, columns, f, turns a workgroup at least
VALUES = {
    "words_one_row": (64, 3, 8, 8, 1, 1, 128, 12000, 9, 4),
    "words_one_row_f0": (64, 2, 8, 8, 1, 1, 64, 12000, 0, 4),
    "words_four_rows": (64, 3, 8, 8, 2, 2, 40, 12003, 9, 4),
    "words_three_rows_f0": (64, 2, 8, 8, 3, 1, 128, 12001, 0, 4),
    "words_five_parties": (64, 5, 8, 8, 1, 2, 64, 12001, 9, 4),
    "words_two_column_blocks": (64, 2, 8, 4, 1, 1, 256, 12001, 9, 4),
    "words32_one_row": (32, 3, 8, 8, 1, 1, 128, 12001, 9, 4),
    "words32_two_rows_f0": (32, 2, 8, 8, 2, 1, 80, 12002, 0, 4),
    "words32_six_parties": (32, 6, 8, 8, 1, 2, 64, 12002, 9, 4),
    "digits_one_tile": (64, 3, 8, 4, 2, 3, 128, 8000, 9, 4),
    "digits_one_tile_f0": (64, 2, 8, 2, 5, 1, 72, 16001, 0, 4),
    "digits_four_waves": (64, 2, 8, 8, 1, 7, 64, 9001, 9, 4),
    "digits_two_tiles": (64, 2, 8, 4, 2, 10, 128, 9000, 9, 4),
    "digits_two_groups": (64, 4, 4, 4, 2, 10, 80, 9002, 9, 4),
    "digits32_one_tile": (32, 3, 8, 8, 2, 4, 128, 8001, 9, 4),
    "digits32_two_tiles": (32, 2, 8, 8, 5, 7, 80, 8002, 9, 4),
    "digits32_four_waves_f0": (32, 2, 8, 8, 1, 9, 40, 16003, 0, 4),
    "digits32_eight_parties": (32, 8, 8, 8, 1, 5, 128, 8001, 9, 4),
}


@pytest.mark.parametrize("name", sorted(VALUES))
def test_values_by_several_turns(name):
    bits, n, batch, kv, share, nodes, dim, columns, f, turns = VALUES[name]
    c = Case(len(name), bits, n, batch, kv, share, nodes, dim, columns)
    lead = (n, batch, c.heads, nodes)
    size = c.ring.cache_values_workspace_bytes(c.pool, c.table, c.heads, nodes, columns)
    ranges = max(1, (size - 256) // (n * batch * c.heads * nodes * dim * bits // 8))
    assert -(-columns // TOKENS) > ranges * (turns - 1), "a workgroup has fewer turns than this case is for"
    P, A, C = words(bits, *lead, columns), words(bits, *lead, columns), words(bits, *lead, dim)
    tup = [words(bits, *lead, dim) for _ in range(3)] if f else None
    seen = c.seen[None, :, None].to(P.dtype)
    want = c.truncated(c.products(P * seen, A * seen, C, False), f, tup)
    got = c.ring.cache_values(c.pool, c.table, c.context, P, A, C, f=f, tuple_=tup, tree=c.tree)
    assert torch.equal(got, want)


def wanted_workgroups():
    with open(os.path.join(build.CSRC, "cache_attention.hip")) as source:
        return int(re.search(r"kScoreWanted = (\d+);", source.read()).group(1))


# bits, n, batch, cached heads, query heads of each, nodes, dim, columns, f, bias, runs a workgroup at least
SCORES = {
    "words_one_row": (64, 3, 8, 8, 1, 1, 64, 6200, 9, True, 3),
    "words_two_rows": (64, 2, 8, 8, 1, 2, 128, 4300, 9, False, 2),
    "words_two_rows_f0": (64, 3, 8, 8, 2, 1, 72, 4300, 0, True, 2),
    "words_five_parties": (64, 5, 8, 8, 1, 1, 64, 4300, 9, True, 2),
    "words32_one_row": (32, 3, 8, 8, 1, 1, 128, 6200, 9, True, 3),
    "words32_two_rows": (32, 4, 8, 8, 2, 1, 40, 4300, 9, True, 2),
    "digits": (64, 3, 8, 8, 2, 2, 64, 6200, 9, True, 3),
    "digits_f0": (64, 2, 8, 8, 1, 3, 128, 4300, 0, True, 2),
    "digits_two_tiles": (64, 2, 8, 4, 4, 5, 40, 6200, 9, True, 3),
    "digits_five_parties": (64, 5, 8, 8, 1, 3, 64, 4300, 9, True, 2),
    "digits_by_k_tiles": (64, 8, 8, 8, 1, 3, 256, 4300, 9, True, 2),
    "digits32": (32, 3, 8, 8, 1, 5, 80, 6200, 9, True, 3),
    "digits32_f0": (32, 2, 8, 8, 3, 1, 64, 4300, 0, False, 2),
    "digits32_eight_parties": (32, 8, 8, 8, 1, 3, 128, 4300, 9, True, 2),
}


@pytest.mark.parametrize("name", sorted(SCORES))
def test_scores_by_several_runs(name):
    bits, n, batch, kv, share, nodes, dim, columns, f, bias, runs = SCORES[name]
    c = Case(len(name), bits, n, batch, kv, share, nodes, dim, columns)
    lead = (n, batch, c.heads, nodes)
    assert -(-columns // TOKENS) * -(-share * nodes // 16) * kv * batch >= runs * wanted_workgroups(), "a workgroup has fewer runs than this case is for"
    Q, A, C = words(bits, *lead, dim), words(bits, *lead, dim), words(bits, *lead, columns)
    tup = [words(bits, *lead, columns) for _ in range(3)] if f else None
    want = c.truncated(c.products(Q, A, C, True), f, tup)
    given = {}
    if bias:
        reach = 150                                           # ends inside a run behind a workgroup's first
        lut, table = spin.relative_buckets(32, reach, False).cuda(), words(bits, n, c.heads, 32)
        at = torch.arange(columns, device="cuda") - c.context[:, None]
        key = torch.where(at < 0, at, c.depth.long().gather(1, at.clamp(0, nodes - 1)))
        away = (key[:, None] - c.depth[:, :, None]).clamp(-reach, reach) + reach
        want = want + table[:, :, lut[away].long()].transpose(1, 2)
        given = dict(bias=(table, lut), depth=c.depth)
    seen = c.seen[:, None]
    want = torch.where(seen, want, torch.zeros((), dtype=want.dtype, device="cuda"))
    want[0] += torch.where(seen, 0, -77).to(want.dtype)
    got = c.ring.cache_scores(c.pool, c.table, c.context, Q, A, C, f=f, tuple_=tup, tree=c.tree, masked=-77, **given)
    assert torch.equal(got, want)


@pytest.mark.parametrize("bits", [64, 32])
@pytest.mark.parametrize("n,nodes,dim,f,bias", [(8, 3, 256, 9, True), (8, 17, 200, 9, False), (5, 4, 256, 0, True), (2, 2, 64, 0, True), (3, 9, 128, 0, True)])
def test_digits_by_k_tiles_and_bias_without_truncation(bits, n, nodes, dim, f, bias):
    """Rows whose digits do not fit LDS at once (eight parties, 64-bit words), on random words; and a bias where nothing is truncated."""
    c = Case(n + nodes, bits, n, 2, 2, 1, nodes, dim, 331, 16)
    lead = (n, 2, 2, nodes)
    Q, A, C = words(bits, *lead, dim), words(bits, *lead, dim), words(bits, *lead, 331)
    tup = [words(bits, *lead, 331) for _ in range(3)] if f else None
    want, given = c.truncated(c.products(Q, A, C, True), f, tup), {}
    if bias:
        lut, table = spin.relative_buckets(16, 40, True).cuda(), words(bits, n, 2, 16)
        at = torch.arange(331, device="cuda") - c.context[:, None]
        key = torch.where(at < 0, at, c.depth.long().gather(1, at.clamp(0, nodes - 1)))
        want = want + table[:, :, lut[(key[:, None] - c.depth[:, :, None]).clamp(-40, 40) + 40].long()].transpose(1, 2)
        given = dict(bias=(table, lut), depth=c.depth)
    seen = c.seen[:, None]
    want = torch.where(seen, want, torch.zeros((), dtype=want.dtype, device="cuda"))
    want[0] += torch.where(seen, 0, 5).to(want.dtype)
    assert torch.equal(c.ring.cache_scores(c.pool, c.table, c.context, Q, A, C, f=f, tuple_=tup, tree=c.tree, masked=5, **given), want)
