"""A block of linear attention on shares, as a program trains and serves it: layer norm, one projection to queries, keys and values, causal attention with a decay for each
head over chunks; all gradients; then tokens one at a time, from the state that the prompt left.

    python examples/block.py

A stand-in, as elsewhere in this repository: one process deals masks, their products and truncation tuples (the paper's offline phase)."""
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))
from paper_2402_02320_amd import spin  # noqa: E402
from generate import Dealer  # noqa: E402

F, G, SHIFT, ITERATIONS = 16, 20, 26, 6    # fractional bits of values, of decay weights, of 1 / dim; Newton's steps
LINE = (3 << (F - 1), 1 << (F - 2))        # the first guess at 1 / sqrt(v), 1.5 - v / 4
EPS = 1                                    # 2^-16


def rates(heads, device):
    return 1 - 2.0 ** -(3 + torch.arange(heads, dtype=torch.float64, device=device))


class Block:
    """Shares of one block's weights and its passes.  Keeps every tensor of its last pass in the open in `seen`, for the comparison with float64."""

    def __init__(self, n, batch, heads, dim, chunk, seed=5):
        self.n, self.batch, self.heads, self.dim, self.chunk, self.width = n, batch, heads, dim, chunk, heads * dim
        self.dealer, self.seen = Dealer(n, seed), {}
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.real = lambda *shape: torch.randn(shape, dtype=torch.float64, device="cuda", generator=g)
        j = torch.arange(chunk + 1, dtype=torch.float64, device="cuda")
        self.decay = torch.round(rates(heads, "cuda")[:, None] ** j * 2 ** G).long()
        self.gamma, self.beta = self.shared("gamma", 1 + 0.1 * self.real(self.width)), self.shared("beta", 0.1 * self.real(self.width))
        self.weights = self.shared("weights", self.real(self.width, 3 * self.width) * 0.5 / self.width ** 0.5)

    # -- dealing ---------------------------------------------------------------------------------------------------
    def shared(self, name, x):
        return self.keep(name, self.dealer.shares(spin.encode(x, F)))

    def keep(self, name, x):
        self.seen[name] = spin.decode(spin.open(x), F)
        return x

    def mask(self, like):
        m = self.dealer.random(*like.shape[1:])
        return m, spin.open(m)

    def product(self, x, y):
        """T(x . y) of shared matrices."""
        (a, A), (b, B) = self.mask(x), self.mask(y)
        z = spin.beaver_matmul(x[:, None], y[:, None], a[:, None], b[:, None], self.dealer.shares(self.dealer.product(A[None], B[None])))[:, 0]
        return spin.trunc(z, *self.dealer.tuple(z.shape[1:]), F)

    def row_words(self, rows, layout):
        """layout: for each word of a row, None (a mask), an int (of a tuple that cuts so many bits: three words) or what is given of the masks, opened, so far."""
        words, opened = [], {}
        for entry in layout:
            if isinstance(entry, int):
                words += self.dealer.tuple((rows,), entry)
            elif entry is None:
                words.append(self.dealer.random(rows))
                opened[len(words) - 1] = spin.open(words[-1])
            else:
                words.append(entry)        # filled in below: it may be made of later masks
        return torch.stack([w if isinstance(w, torch.Tensor) else self.dealer.shares(w(opened)) for w in words], 1), opened

    # -- layer norm ------------------------------------------------------------------------------------------------
    def norm(self, x):
        (a, A), (b, B) = self.mask(x), self.mask(x)
        layout = [SHIFT, lambda m: (A * A).sum(-1), F, SHIFT, F, None]
        for k in range(14, 14 + 15 * ITERATIONS, 15):
            layout += [None, lambda m, k=k: m[k] * m[k], F, None, lambda m, k=k: m[k + 5] * m[13], F, None, lambda m, k=k: m[k] * m[k + 10], F + 1]
        words, opened = self.row_words(x.shape[1], layout + [None])
        self.gamma_mask = self.mask(self.gamma)
        C = (self.dealer.shares(A * opened[words.shape[1] - 1][:, None]), self.dealer.shares(B * self.gamma_mask[1]))
        tuples = [self.dealer.tuple(A.shape) for _ in range(2)]
        y, xhat, rstd = spin.layernorm(x, (self.gamma, self.gamma_mask[0]), self.beta, (a, b), C, tuples, words, F, SHIFT, LINE, EPS)
        self.keep("xhat", xhat), self.keep("rstd", rstd)
        return self.keep("y", y), (xhat, (b, B), rstd)

    def norm_grad(self, dy, kept):
        (xhat, (b, B), rstd), (a, A), (c, C) = kept, self.mask(dy), self.mask(dy)
        layout = [SHIFT, lambda m: (C * B).sum(-1), F, SHIFT, None, None, lambda m: m[11] * m[10], F, None, lambda m: m[16] * m[10], F, None]
        words, opened = self.row_words(dy.shape[1], layout)
        columns = torch.stack([self.dealer.shares((A * B).sum(0))] + self.dealer.tuple((self.width,)), 1)
        dealt = (self.dealer.shares(A * self.gamma_mask[1]), self.dealer.shares(C * opened[10][:, None] - B * opened[21][:, None]))
        dx, dgamma, dbeta = spin.layernorm_grad(dy, xhat, rstd, (self.gamma, self.gamma_mask[0]), (a, b, c), dealt, [self.dealer.tuple(A.shape) for _ in range(2)], words,
                                                columns, F, SHIFT)
        return self.keep("dx", dx), self.keep("dgamma", dgamma), self.keep("dbeta", dbeta)

    # -- attention ---------------------------------------------------------------------------------------------------
    def lengths_are(self, tokens, lengths):
        """What the dealer's sums over chunks need: which tokens of a chunk are there, and their weights."""
        self.tokens, self.chunks = tokens, -(-tokens // self.chunk)
        self.lengths = torch.tensor(lengths, dtype=torch.int32, device="cuda")
        i = torch.arange(self.chunk, device="cuda")
        L = (self.lengths.long()[:, None] - self.chunk * torch.arange(self.chunks, device="cuda")).clamp(0, self.chunk)       # [batch, chunks]
        self.there = (i < L[..., None])[:, None, ..., None]                                              # [batch, 1, chunks, chunk, 1]
        self.near = self.decay[:, (i[:, None] - i).clamp(min=0)][None, :, None]
        self.to_end = self.decay[:, (L[..., None] - 1 - i).clamp(min=0)].transpose(0, 1)[..., None]      # [batch, heads, chunks, chunk, 1]
        self.from_start = self.decay[:, i + 1][None, :, None, :, None].expand_as(self.to_end)
        self.call = dict(f=F, g=G, decay=self.decay, lengths=self.lengths)

    def by_chunk(self, x):
        x = torch.nn.functional.pad(x, (0, 0, 0, self.chunks * self.chunk - x.shape[-2]))
        return x.reshape(x.shape[:-2] + (self.chunks, self.chunk, x.shape[-1])) * self.there

    def opened(self, x, y, transposed=False):
        """x . y of all chunks' matrices, in the open."""
        lead = x.shape[:-2]
        return self.dealer.product(x.flatten(0, -3).contiguous(), y.flatten(0, -3).contiguous(), transposed).unflatten(0, lead)

    def scores(self, x, y):
        C = self.near * self.opened(self.by_chunk(x[2]), self.by_chunk(y[2]), True)
        return spin.linattn_scores(x[:2], y[:2], self.dealer.shares(C), self.dealer.tuple(C.shape, F + G), **self.call)

    def states(self, x, y, first=None, reverse=False):
        X = self.by_chunk(x[2]) * (self.from_start if reverse else self.to_end)
        C = self.opened(X.transpose(-1, -2), self.by_chunk(y[2]))
        return spin.linattn_states(x[:2], y[:2], self.dealer.shares(C), self.dealer.tuple(C.shape, F + G), chunk=self.chunk, first=first, reverse=reverse, **self.call)

    def outputs(self, P, y, x, S, reverse=False, transposed=False):
        p = P[2].tril()
        C = self.opened(p.transpose(-1, -2) if reverse else p, self.by_chunk(y[2])) << G
        C = C + self.opened(self.by_chunk(x[2]) * (self.to_end if reverse else self.from_start), S[2], transposed)
        C = C.flatten(2, 3)[:, :, :self.tokens]
        return spin.linattn_outputs(P[:2], y[:2], x[:2], S[:2], self.dealer.shares(C), self.dealer.tuple(C.shape, F + G), reverse=reverse, transposed=transposed, **self.call)

    def factor(self, x):
        """Shares, their masks, and the masks in the open."""
        return (x,) + self.mask(x)

    def heads_of(self, qkv):
        """[n, batch * tokens, 3 width] -> queries, keys and values, [n, batch, heads, tokens, dim]."""
        return [t.contiguous() for t in qkv.view(self.n, self.batch, -1, 3, self.heads, self.dim).permute(3, 0, 1, 4, 2, 5)]

    # -- passes ------------------------------------------------------------------------------------------------------
    def forward(self, x, lengths):
        """x: shares of [batch * tokens, width] -> (output, the state behind the last token, what the backward pass takes)."""
        self.lengths_are(x.shape[1] // self.batch, lengths)
        y, of_norm = self.norm(x)
        qkv = self.product(y, self.weights)
        q, k, v = [self.factor(self.keep(name, t)) for name, t in zip("qkv", self.heads_of(qkv))]
        P = self.factor(self.scores(q, k))
        S, last = self.states(k, v)
        S = self.factor(S)
        return self.keep("o", self.outputs(P, v, q, S)), self.keep("last", last), (y, of_norm, q, k, v, P, S)

    def backward(self, do, kept):
        """Gradients of x, gamma, beta and the projection, from shares of the output's."""
        y, of_norm, q, k, v, P, S = kept
        do = self.factor(do)
        dP = self.factor(self.scores(do, v))
        dS = self.factor(self.states(q, do, reverse=True)[0])
        dq = self.outputs(dP, k, do, S, transposed=True)
        dk = self.outputs(dP, q, v, dS, reverse=True, transposed=True)
        dv = self.outputs(P, do, k, dS, reverse=True)
        for name, t in zip(("dq", "dk", "dv"), (dq, dk, dv)):
            self.keep(name, t)
        dqkv = torch.stack([dq, dk, dv]).permute(1, 2, 4, 0, 3, 5).reshape(self.n, -1, 3 * self.width)
        self.keep("dqkv", dqkv)
        self.keep("dweights", self.product(y.transpose(1, 2).contiguous(), dqkv))
        dy = self.keep("dy", self.product(dqkv, self.weights.transpose(1, 2).contiguous()))
        return self.norm_grad(dy, of_norm)

    def token(self, x, state, active=None):
        """One token of each sequence: x, shares of [batch, width] -> (output [batch, heads, dim], state); sequences that are not active keep theirs."""
        y, _ = self.norm(x)
        q, k, v = [self.factor(self.keep(name, t[..., 0, :].contiguous())) for name, t in zip("qkv", self.heads_of(self.product(y, self.weights)))]
        m, M = self.mask(state)
        C = (self.decay[:, 0, None, None] * (k[2][..., None] * v[2][..., None, :]), (q[2][..., None] * M).sum(-2))
        tuples = (self.dealer.tuple(C[0].shape, F + G), self.dealer.tuple(C[1].shape))
        out, state = spin.linattn_step(state, q[:2], k[:2], v[:2], m, [self.dealer.shares(c) for c in C], tuples, F, self.decay[:, :2].contiguous(), G, active)
        return self.keep("o", out), self.keep("last", state)


def norm(x, gamma, beta):
    """Layer norm in float64."""
    c = x - x.mean(-1, keepdim=True)
    return c / (c.square().mean(-1, keepdim=True) + EPS * 2.0 ** -F).sqrt() * gamma + beta


def attention(q, k, v, lengths, state=None):
    """Its recurrence in float64: S <- rate S + k (x) v, o = q . S."""
    rate = rates(q.shape[1], q.device)[:, None, None]
    S = torch.zeros(q.shape[:2] + (k.shape[-1], v.shape[-1]), dtype=q.dtype, device=q.device) if state is None else state
    out = []
    for t in range(q.shape[2]):
        there = torch.tensor([t < n for n in lengths], device=q.device)[:, None, None, None]
        S = torch.where(there, rate * S + k[:, :, t, :, None] * v[:, :, t, None], S)
        out.append(torch.where(there[..., 0], (q[:, :, t, :, None] * S).sum(-2), 0))
    return torch.stack(out, 2), S


def split(qkv, batch, heads, dim):
    return qkv.view(batch, -1, 3, heads, dim).permute(2, 0, 3, 1, 4)


if __name__ == "__main__":
    n, heads, dim, chunk, lengths = 3, 2, 32, 32, [70, 33]
    block = Block(n, len(lengths), heads, dim, chunk)
    tokens, width = max(lengths), heads * dim
    x, do = block.real(len(lengths) * tokens, width), block.real(len(lengths), heads, tokens, dim)
    _, state, kept = block.forward(block.shared("x", x), lengths)
    block.backward(block.shared("do", do), kept)
    leaves = [t.requires_grad_() for t in (x, block.seen["gamma"].clone(), block.seen["beta"].clone(), block.seen["weights"].clone())]
    o, S = attention(*split(norm(*leaves[:3]) @ leaves[3], len(lengths), heads, dim), lengths)
    (o * do).sum().backward()
    S = S.detach()
    for name, want in [("o", o.detach()), ("last", S)] + list(zip(("dx", "dgamma", "dbeta", "dweights"), [t.grad for t in leaves])):
        print("%-8s on shares against float64: largest difference %.2g of %.3g" % (name, (block.seen[name] - want).abs().max().item(), want.abs().max().item()))
    gamma, beta, weights = [t.detach() for t in leaves[1:]]
    for step in range(3):
        x = block.real(len(lengths), width)
        _, state = block.token(block.shared("x", x), state)
        o, S = attention(*split(norm(x, gamma, beta) @ weights, len(lengths), heads, dim), [1] * len(lengths), S)
        print("token %d on shares against float64: largest difference %.2g of %.3g" % (step, (block.seen["o"] - o[:, :, 0]).abs().max().item(), o.abs().max().item()))
