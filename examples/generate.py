"""Attention of a generating transformer on shares, as a program runs it: prompts enter the paged cache, a tree of drafted tokens is scored over it with a learned
relative position bias, its values are summed, the accepted branch is kept, a sequence forks, and the bias takes training steps.

    python examples/generate.py

Stand-ins, as elsewhere in this repository: one process deals triples and truncation tuples (the paper's offline phase), and softmax, which the paper's parties compute by
comparisons and polynomials between the two products, is done here on opened scores and shared again.  Every result is compared with float64 attention."""
import math
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2402_02320_amd import spin  # noqa: E402
from paper_2402_02320_amd.cache import ShareCache  # noqa: E402

F = 16                                     # fractional bits
NOTHING = -(1 << 40)                       # what a score is where nothing is seen: -2^24


class Dealer:
    """Masks, triples and truncation tuples, drawn from the library's counter generator."""

    def __init__(self, n, seed):
        self.n, self.seed, self.stream = n, seed, 100

    def shares(self, x):
        self.stream += 1
        return spin.share(x.contiguous(), self.n, self.seed, self.stream)

    def random(self, *shape):
        self.stream += 1
        return torch.stack([spin.random(math.prod(shape), self.seed, self.stream, i).view(shape) for i in range(self.n)])

    def tuple(self, shape, f=F):
        r = spin.open(self.random(*shape))
        return [self.shares(t) for t in (r, (r >> f) & ((1 << (63 - f)) - 1), (r >> 63) & 1)]

    @staticmethod
    def product(x, y, transposed=False):
        """x . y (or x . y^T) of ring matrices in the open: a Beaver product of one party without masks."""
        x, y = x[None], y[None]
        none = torch.zeros_like
        c = torch.zeros(x.shape[:3] + (y.shape[2 if transposed else 3],), dtype=torch.int64, device=x.device)
        return spin.beaver_matmul(x, y, none(x), none(y), c, y_transposed=transposed)[0]


def attend(dealer, cache, seqs, q, masks, tree, depth, bias):
    """q: float64 [batch, heads, nodes, dim]; masks: {sequence: (opened masks of its K rows, of its V rows)} -> attention output, float64."""
    n, (batch, heads, nodes, dim) = dealer.n, q.shape
    cached = cache.pools[0].shape[2]
    group = heads // cached
    columns = max(cache.length(s) for s in seqs)
    table, context = cache.table(seqs), cache.context(seqs, nodes)

    def dealt(kind):                       # the masks of all cached rows, [batch * heads, columns, dim]
        m = torch.zeros(batch, cached, columns, dim, dtype=torch.int64, device=q.device)
        for k, s in enumerate(seqs):
            m[k, :, :cache.length(s)] = masks[s][kind]
        return m.repeat_interleave(group, 1).reshape(batch * heads, columns, dim)
    A = dealer.random(batch, heads, nodes, dim)
    C = dealer.shares(dealer.product(spin.open(A).view(-1, nodes, dim), dealt(0), transposed=True).view(batch, heads, nodes, columns))
    Q = dealer.shares(spin.encode(q, F))
    S = spin.cache_scores(cache.pools[0], table, context, Q, A, C, f=F, tuple_=dealer.tuple((batch, heads, nodes, columns)), tree=tree, masked=NOTHING, bias=bias, depth=depth)
    P = torch.softmax(spin.decode(spin.open(S), F), -1)                                        # stand-in for the protocol
    at = torch.arange(columns, device=q.device) - context[:, None, None]                       # what is seen, for the dealer's sums
    seen = (at < 0) | ((at < nodes) & ((tree[:, :, None] >> at.clamp(0, nodes - 1)) & 1 > 0))
    A = dealer.random(batch, heads, nodes, columns)
    opened = torch.where(seen[:, None], spin.open(A), 0).view(-1, nodes, columns)
    C = dealer.shares(dealer.product(opened, dealt(1)).view(batch, heads, nodes, dim))
    O = spin.cache_values(cache.pools[1], table, context, dealer.shares(spin.encode(P, F)), A, C, f=F, tuple_=dealer.tuple((batch, heads, nodes, dim)), tree=tree)
    return spin.decode(spin.open(O), F), spin.decode(spin.open(S), F)


def reference(q, k, v, group, seen, bias):
    """float64 attention of one sequence: q [heads, nodes, dim], k, v [cached heads, rows, dim], seen [nodes, rows], bias [heads, nodes, rows]."""
    k, v = k.repeat_interleave(group, 0), v.repeat_interleave(group, 0)
    s = torch.where(seen, (q[..., None, :] * k[:, None]).sum(-1) + bias, -2.0 ** 24)
    return (torch.softmax(s, -1)[..., None] * v[:, None]).sum(-2)


def generate(n=3, heads=8, cached=2, dim=64, prompts=(70, 33), steps=3):
    dev, g = "cuda", torch.Generator(device="cuda").manual_seed(1)

    def real(*shape):
        return torch.randn(shape, dtype=torch.float64, device=dev, generator=g)
    dealer, cache = Dealer(n, 77), ShareCache(n, 32, cached, dim, page_tokens=16)
    lut, table = spin.relative_buckets(32, 64, False).to(dev), real(heads, 32) * 0.1
    bias = (dealer.shares(spin.encode(table, F)), lut)
    plain, masks = {}, {}                  # what the cache holds, in the open, and the dealer's masks

    def append(seqs, rows, counts):
        k, v = real(len(seqs), cached, rows, dim) * 0.3, real(len(seqs), cached, rows, dim)
        b = [dealer.random(len(seqs), cached, rows, dim) for _ in range(2)]
        cache.append(seqs, [dealer.shares(spin.encode(t, F)) for t in (k, v)], b, counts)
        opened = [spin.open(t) for t in b]
        for j, (s, c) in enumerate(zip(seqs, counts)):
            for store, new in ((plain, (k, v)), (masks, opened)):
                old = store.get(s, [t[j, :, :0] for t in new])
                store[s] = [torch.cat([o, t[j, :, :c]], 1) for o, t in zip(old, new)]
    seqs = [cache.add() for _ in prompts]
    append(seqs, max(prompts), list(prompts))
    worst = 0.0
    parent = [-1, 0, 0, 1, 2, 4]           # the drafted tree
    sees, deep = [], []
    for j, p in enumerate(parent):
        sees.append((sees[p] if p >= 0 else 0) | 1 << j)
        deep.append(deep[p] + 1 if p >= 0 else 0)
    nodes = len(parent)
    for step in range(steps):
        if step == 1:                      # a second continuation of the first prompt
            seqs.append(cache.fork(seqs[0]))
            plain[seqs[-1]], masks[seqs[-1]] = list(plain[seqs[0]]), list(masks[seqs[0]])
        append(seqs, nodes, [nodes] * len(seqs))
        tree = torch.tensor([sees] * len(seqs), dtype=torch.int64, device=dev)
        depth = torch.tensor([deep] * len(seqs), dtype=torch.int32, device=dev)
        q = real(len(seqs), heads, nodes, dim) * 0.3
        got, _ = attend(dealer, cache, seqs, q, masks, tree, depth, bias)
        for j, s in enumerate(seqs):
            rows = cache.length(s)
            at = torch.arange(rows, device=dev) - (rows - nodes)
            seen = (at < 0) | ((tree[j][:, None] >> at.clamp(min=0)) & 1 > 0)
            place = torch.where(at < 0, at, depth[j].long()[at.clamp(min=0)])
            away = (place - depth[j].long()[:, None]).clamp(-64, 64) + 64
            want = reference(q[j], *plain[s], heads // cached, seen, table[:, lut[away].long()])
            worst = max(worst, float((got[j] - want).abs().max()))
        kept = [[0, 2, 4, 5] if (step + j) % 2 else [0, 1, 3] for j in range(len(seqs))]       # a branch of the tree, as a model would accept it
        cache.keep(seqs, nodes, kept)
        for s, k in zip(seqs, kept):
            for store in (plain, masks):
                store[s] = [torch.cat([t[:, :-nodes], t[:, -nodes:][:, k]], 1) for t in store[s]]
    cache.free(seqs[1])
    used = cache.compact()
    return worst, used


def train_bias(n=3, batch=2, heads=4, tokens=40, steps=8, rate=0.9):
    """The bias learns target scores on shares: loss = mean over what is seen of (scores + bias - target)^2 / 2."""
    dev, g = "cuda", torch.Generator(device="cuda").manual_seed(2)
    dealer = Dealer(n, 78)
    lut = spin.relative_buckets(16, 32, False).to(dev)
    scores = torch.randn(batch, heads, tokens, tokens, dtype=torch.float64, device=dev, generator=g)
    hidden = torch.randn(heads, 16, dtype=torch.float64, device=dev, generator=g)
    away = (torch.arange(tokens, device=dev) - torch.arange(tokens, device=dev)[:, None]).clamp(-32, 32) + 32
    target = scores + hidden[:, lut[away].long()]
    X, Y = dealer.shares(spin.encode(scores, F) << F), dealer.shares(spin.encode(target, F))   # scores as a product leaves them, at 2 F
    table = dealer.shares(torch.zeros(heads, 16, dtype=torch.int64, device=dev))
    lengths = torch.tensor([tokens, tokens - 7], dtype=torch.int32, device=dev)
    # the places of the bucket that has most of them: no bucket's step goes past its target
    count = torch.bincount(lut[away][torch.tril(torch.ones(tokens, tokens, dtype=torch.bool, device=dev))].long(), minlength=16).clamp(min=1).max().item() * batch
    losses = []
    for _ in range(steps):
        S = spin.relbias_trunc(X, table, lut, f=F, tuple_=dealer.tuple(scores.shape), causal=True, lengths=lengths)
        dS = S - Y                         # local to every party; masked places take no part in the gradient
        grad = spin.relbias_grad(dS, lut, 16, causal=True, lengths=lengths)
        table = spin.lincomb_trunc([table, grad], [1 << F, -int(rate / count * 2 ** F)], f=F, tuple_=dealer.tuple((heads, 16)))
        losses.append(float((spin.decode(spin.open(table), F) - hidden).abs().max()))
    return losses


if __name__ == "__main__":
    worst, used = generate()
    print("drafted attention on shares against float64: largest difference %.2g; %d pages in use after compaction" % (worst, used))
    print("largest distance of the learned bias from the hidden one, by step:", " ".join("%.3f" % v for v in train_bias()))
