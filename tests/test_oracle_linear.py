"""What the oracle of linear attention and layer norm computes, on dealt masks: linear attention with a decay and its gradients, layer norm and its gradients, in float64 and
by differences.  On the CPU."""
import numpy as np
import pytest

from oracle import linear as lin

F, G, N = 16, 12, 3


class Dealer:
    """Shares, masks and tuples from numpy's generator; 64-bit words."""

    def __init__(self, seed):
        self.rng = np.random.default_rng(seed)

    def words(self, *shape):
        return self.rng.integers(0, 1 << 64, size=shape, dtype=np.uint64)

    def shares(self, x):
        rest = self.words(N - 1, *x.shape)
        return np.concatenate([(x - rest.sum(0, dtype=np.uint64))[None], rest])

    def encode(self, x):
        return self.shares(np.floor(np.asarray(x) * 2.0 ** F).astype(np.int64).view(np.uint64))

    def masked(self, shares):
        return shares, self.words(*shares.shape)

    def tuple(self, shape, f):
        r = self.words(*shape)
        return [self.shares(t) for t in (r, (r >> np.uint64(f)) & np.uint64((1 << (63 - f)) - 1), r >> np.uint64(63))]


def value(shares, f=F):
    return shares.sum(0, dtype=np.uint64).view(np.int64) / 2.0 ** f


def mask_of(x):
    """The mask of a factor, in the open."""
    return x[1].sum(0, dtype=np.uint64)


class Attention:
    def __init__(self, seed, batch=2, heads=2, tokens=19, dk=4, dv=3, chunk=8, lengths=(19, 11)):
        self.d, self.chunk, self.lengths = Dealer(seed), chunk, np.array(lengths)
        self.shape, self.chunks = (batch, heads, tokens, dk, dv), -(-tokens // chunk)
        self.decay = np.array([[round((1 - 2.0 ** -(3 + h)) ** j * 2 ** G) for j in range(chunk + 1)] for h in range(heads)], np.uint64)
        self.kw = dict(f=F, decay=self.decay, g=G, lengths=self.lengths)

    def parts(self):
        batch, heads, tokens, _, _ = self.shape
        for b, c, rows in lin.chunks_of(tokens, self.chunk, self.lengths, batch):
            for h in range(heads):
                yield b, h, c, rows, rows.stop - rows.start, self.decay[h]

    def scores(self, x, y):
        C = np.zeros(self.shape[:2] + (self.chunks, self.chunk, self.chunk), np.uint64)
        for b, h, c, rows, L, w in self.parts():
            i, j = np.indices((L, L))
            C[b, h, c, :L, :L] = w[np.maximum(i - j, 0)] * (mask_of(x)[b, h, rows] @ mask_of(y)[b, h, rows].T)
        return lin.scores(x, y, self.d.shares(C), self.d.tuple(C.shape, F + G), **self.kw)

    def states(self, x, y, first, reverse=False):
        C = np.zeros(self.shape[:2] + (self.chunks, x[0].shape[-1], y[0].shape[-1]), np.uint64)
        for b, h, c, rows, L, w in self.parts():
            C[b, h, c] = (mask_of(x)[b, h, rows] * (w[1:L + 1] if reverse else w[:L][::-1])[:, None]).T @ mask_of(y)[b, h, rows]
        return lin.states(x, y, self.d.shares(C), self.d.tuple(C.shape, F + G), chunk=self.chunk, first=first, reverse=reverse, **self.kw)

    def outputs(self, P, y, x, S, reverse=False, transposed=False):
        C = np.zeros(self.shape[:3] + (y[0].shape[-1],), np.uint64)
        for b, h, c, rows, L, w in self.parts():
            p, s = mask_of(P)[b, h, c, :L, :L] * np.tri(L, dtype=np.uint64), mask_of(S)[b, h, c]
            C[b, h, rows] = ((p.T if reverse else p) @ mask_of(y)[b, h, rows] << np.uint64(G)) + \
                (mask_of(x)[b, h, rows] * (w[:L][::-1] if reverse else w[1:L + 1])[:, None]) @ (s.T if transposed else s)
        return lin.outputs(P, y, x, S, self.d.shares(C), self.d.tuple(C.shape, F + G), reverse=reverse, transposed=transposed, **self.kw)

    def real(self, q, k, v, first):
        """(results, last states) in float64, token by token; the decay over a whole chunk is the table's."""
        batch, heads, tokens, _, dv = self.shape
        out, last = np.zeros((batch, heads, tokens, dv)), first.copy()
        for b in range(batch):
            for h in range(heads):
                w = self.decay[h] / 2.0 ** G
                for c in range(self.chunks):
                    rows = range(c * self.chunk, max(c * self.chunk, min((c + 1) * self.chunk, int(self.lengths[b]))))
                    S, L = last[b, h].copy(), len(rows)
                    for i, t in enumerate(rows):
                        out[b, h, t] = w[i + 1] * q[b, h, t] @ S + sum(w[i - j] * (q[b, h, t] @ k[b, h, r]) * v[b, h, r] for j, r in enumerate(rows[:i + 1]))
                    if L:
                        last[b, h] = w[L] * S + sum(w[L - 1 - j] * np.outer(k[b, h, r], v[b, h, r]) for j, r in enumerate(rows))
        return out, last


# Sizes below are at most one.  Encoding moves a factor by less than u = 2^-16, truncation a result by at most u.  Within a chunk of 8: a score (4 terms) is off by (4 * 2 + 1) u,
# a state of at most three chunks (19 tokens of sizes up to 1 * 1) by (19 * 2 + 3) u.  A result: 8 scores of sizes up to 4 times values, 8 (9 + 4) u; queries times states of sizes up to
# 19 and off as above, 4 (19 + 41) u; and its truncation: less than 512 u.  Gradients are sums of the same lengths with the result's gradient in the place of one factor.
FORWARD = 512 * 2.0 ** -F


def test_attention_and_its_gradients():
    a = Attention(1)
    batch, heads, tokens, dk, dv = a.shape
    rng = np.random.default_rng(2)
    q, k, v, dO, dlast, first = (rng.uniform(-1, 1, s) for s in [(batch, heads, tokens, dk)] * 2 + [(batch, heads, tokens, dv)] * 2 + [(batch, heads, dk, dv)] * 2)
    Q, K, V, DO = (a.d.masked(a.d.encode(x)) for x in (q, k, v, dO))
    P = a.d.masked(a.scores(Q, K))
    states, last = a.states(K, V, a.d.encode(first))
    S = a.d.masked(states)
    out = a.outputs(P, V, Q, S)
    want, want_last = a.real(q, k, v, first)
    assert np.abs(value(out) - want).max() < FORWARD and np.abs(value(last) - want_last).max() < FORWARD
    dP = a.d.masked(a.scores(DO, V))
    back, dfirst = a.states(Q, DO, a.d.encode(dlast), reverse=True)
    dS = a.d.masked(back)
    grads = dict(q=a.outputs(dP, K, DO, S, transposed=True), k=a.outputs(dP, Q, V, dS, reverse=True, transposed=True), v=a.outputs(P, DO, K, dS, reverse=True), first=dfirst)
    # by differences: the results are linear in each factor by itself, so that a step of one shows the derivative up to float64's rounding
    point = dict(q=q, k=k, v=v, first=first)

    def total(p):
        o, l = a.real(**p)
        seen = np.arange(tokens) < a.lengths[:, None]
        return (o * dO)[np.broadcast_to(seen[:, None], o.shape[:3])].sum() + (l * dlast).sum()
    base = total(point)
    for name, g in grads.items():
        for at in [tuple(rng.integers(0, s) for s in point[name].shape) for _ in range(25)]:
            moved = point[name].copy()
            moved[at] += 1
            assert abs(value(g)[at] - (total(dict(point, **{name: moved})) - base)) < 4 * FORWARD, (name, at)
    for name in "qkv":                                        # what is not there has no gradient
        assert (value(grads[name])[1, :, 11:] == 0).all()


def test_steps_are_the_chunked_form():
    """Single tokens from a prompt's last state on, against the float64 recurrence."""
    a = Attention(3, tokens=8, lengths=(8, 8))
    batch, heads, tokens, dk, dv = a.shape
    rng = np.random.default_rng(4)
    q, k, v, first = (rng.uniform(-1, 1, s) for s in [(batch, heads, tokens, dk)] * 2 + [(batch, heads, tokens, dv), (batch, heads, dk, dv)])
    S, real, w = a.d.encode(first), first.copy(), a.decay[:, :2]
    for t in range(tokens):
        Q, K, V = (a.d.masked(a.d.encode(x[:, :, t])) for x in (q, k, v))
        mask = a.d.words(*S.shape)
        CS = w[None, :, 0, None, None] * mask_of(K)[..., None] * mask_of(V)[:, :, None]
        CO = (mask_of(Q)[..., None] * mask.sum(0, dtype=np.uint64)).sum(-2, dtype=np.uint64)
        out, S = lin.step(S, Q, K, V, mask, (a.d.shares(CS), a.d.shares(CO)), (a.d.tuple(CS.shape, F + G), a.d.tuple(CO.shape, F)), F, w, G)
        lam = (w / 2.0 ** G)[None, :, :, None, None]
        real = lam[:, :, 1] * real + lam[:, :, 0] * k[:, :, t, :, None] * v[:, :, t, None]
        # eight steps of (2 + 1) u, times four terms of sizes up to one, and the queries' roundings on states of sizes up to nine
        assert np.abs(value(S) - real).max() < 25 * 2.0 ** -F
        assert np.abs(value(out) - (q[:, :, t, None] @ real)[:, :, 0]).max() < (4 * (25 + 9) + 1) * 2.0 ** -F


SHIFT, LINE, EPS, ITERATIONS = 26, (3 << (F - 1), 1 << (F - 2)), 1, 6


def newton_words(d, rows, iterations):
    """Row words [n, 15 (iterations + 1), rows] of the forward pass, and the last of them."""
    r = {}

    def put(k, x):
        r[k] = x

    def cut(k, f):
        for j, t in enumerate(d.tuple((rows,), f)):
            put(k + j, t)
    cut(0, SHIFT)
    cut(4, F)
    cut(7, SHIFT)
    cut(10, F)
    v = d.words(rows)
    put(13, d.shares(v))
    for k in range(14, 14 + 15 * iterations, 15):
        y, u, h = d.words(rows), d.words(rows), d.words(rows)
        for at, x in ((0, y), (1, y * y), (5, u), (6, u * v), (10, h), (11, y * h)):
            put(k + at, d.shares(x))
        cut(k + 2, F)
        cut(k + 7, F)
        cut(k + 12, F + 1)
    last = d.words(rows)
    put(14 + 15 * iterations, d.shares(last))
    return r, last


def test_norm_and_its_gradients():
    d, rows, dim = Dealer(5), 6, 16
    rng = np.random.default_rng(6)
    x, gamma, beta, dy = rng.uniform(-2, 2, (rows, dim)), rng.uniform(-1.5, 1.5, dim), rng.uniform(-1, 1, dim), rng.uniform(-1, 1, (rows, dim))
    x -= rng.uniform(-3, 3, (rows, 1))                        # means and variances differ from row to row
    x *= rng.uniform(0.6, 1.2, (rows, 1))
    X, GAMMA = d.encode(x), d.masked(d.encode(gamma))
    words, b = newton_words(d, rows, ITERATIONS)
    m1, m2 = d.words(N, rows, dim), d.words(N, rows, dim)
    o1, o2 = m1.sum(0, dtype=np.uint64), m2.sum(0, dtype=np.uint64)
    words[3] = d.shares((o1 * o1).sum(-1, dtype=np.uint64))
    row_words = np.stack([words[k] for k in range(15 * (ITERATIONS + 1))], 1)
    y, xhat, rstd = lin.layernorm(X, GAMMA, d.encode(beta), (m1, m2), (d.shares(o1 * b[:, None]), d.shares(o2 * mask_of(GAMMA))),
                                  (d.tuple((rows, dim), F), d.tuple((rows, dim), F)), row_words, F, SHIFT, LINE, EPS)

    def norm(x, gamma, beta):
        c = x - x.mean(-1, keepdims=True)
        r = 1 / np.sqrt((c * c).mean(-1, keepdims=True) + EPS * 2.0 ** -F)
        return c * r * gamma + beta, c * r, r[:, 0]
    want = norm(x, gamma, beta)
    # u = 2^-16.  Means are off by 2 u, centred words (sizes up to 6) by 4 u, the variance (0.3 to 3) by 2 * 6 * 4 u + 3 u; 1 / sqrt of it (up to 2) by half of 2^3 of that, and by
    # Newton's own roundings, less than 8 u: 212 u; normed words (up to 4) by 6 * 212 u + 4 * 2 u + u; the result by 1.5 times that and 4 u + 2 u.
    u = 2.0 ** -F
    assert np.abs(value(rstd) - want[2]).max() < 212 * u and np.abs(value(xhat) - want[1]).max() < 1300 * u and np.abs(value(y) - want[0]).max() < 2000 * u
    # backward
    g_words = {}

    def cut(k, f):
        for j, t in enumerate(d.tuple((rows,), f)):
            g_words[k + j] = t
    a1, a3 = d.words(N, rows, dim), d.words(N, rows, dim)
    p1, p3 = a1.sum(0, dtype=np.uint64), a3.sum(0, dtype=np.uint64)
    am1, am2, ak = d.words(rows), d.words(rows), d.words(rows)
    for k, f in ((0, SHIFT), (4, F), (7, SHIFT), (13, F), (18, F)):
        cut(k, f)
    for k, v in ((3, (p3 * o2).sum(-1, dtype=np.uint64)), (10, b), (11, am1), (12, am1 * b), (16, am2), (17, am2 * b), (21, ak)):
        g_words[k] = d.shares(v)
    columns = np.stack([d.shares((p1 * o2).sum(0, dtype=np.uint64))] + d.tuple((dim,), F), 1)
    dx, dgamma, dbeta = lin.layernorm_grad(d.encode(dy), xhat, rstd, GAMMA, (a1, m2, a3), (d.shares(p1 * mask_of(GAMMA)), d.shares(p3 * b[:, None] - o2 * ak[:, None])),
                                           (d.tuple((rows, dim), F), d.tuple((rows, dim), F)), np.stack([g_words[k] for k in range(22)], 1), columns, F, SHIFT)

    def total(x, gamma, beta):
        return (norm(x, gamma, beta)[0] * dy).sum()
    h = 1e-5                                                  # central differences: their own error is below 1e-8 here
    # sums of six rows of normed words off as above; of dx's three terms (sizes up to 3, 3, 4 * 4) each product's two factors are off by at most 1300 u times 4
    for name, got, bound in (("beta", dbeta, 6 * u), ("gamma", dgamma, 6 * 1310 * u), ("x", dx, 3 * 4 * 1300 * u)):
        point = dict(x=x, gamma=gamma, beta=beta)
        for at in np.ndindex(point[name].shape):
            up, down = point[name].copy(), point[name].copy()
            up[at] += h
            down[at] -= h
            slope = (total(**dict(point, **{name: up})) - total(**dict(point, **{name: down}))) / (2 * h)
            assert abs(value(got)[at] - slope) < bound + 1e-7, (name, at)


@pytest.mark.parametrize("bits", [64, 32])
def test_sums_wrap_at_the_words_width(bits):
    dtype = np.dtype(np.uint64 if bits == 64 else np.uint32)
    x = np.array([[1 << (bits - 1)], [1 << (bits - 1)]], dtype)
    assert lin.opened((x, np.zeros_like(x)))[0] == 0 and lin.inverse(bits - 6, 3, dtype) == ((1 << (bits - 6)) + 1) // 3
