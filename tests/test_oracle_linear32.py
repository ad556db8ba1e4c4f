"""What the oracle of linear attention and layer norm means over Z_2^32, where few bits are left for fractions: against float64 and by differences, within what roundings of the words
add up to.  Values stay where truncation is exact up to one last bit: a sum before it is below 2^30, so at 9 and 6 fractional bits results of attention are below 64, and squares' sums
of a norm at f bits below 2^(30 - 2 f).  On the CPU."""
import numpy as np
import pytest

from oracle import linear as lin

N, WORD = 3, np.uint32


class Dealer:
    """Shares, masks and tuples of 32-bit words from numpy's generator."""

    def __init__(self, seed, f):
        self.rng, self.f = np.random.default_rng(seed), f

    def words(self, *shape):
        return self.rng.integers(0, 1 << 32, size=shape, dtype=WORD)

    def shares(self, x):
        rest = self.words(N - 1, *x.shape)
        return np.concatenate([(x - rest.sum(0, dtype=WORD))[None], rest])

    def encode(self, x):
        return self.shares(np.floor(np.asarray(x) * 2.0 ** self.f).astype(np.int32).view(WORD))

    def masked(self, shares):
        return shares, self.words(*shares.shape)

    def tuple(self, shape, f):
        r = self.words(*shape)
        return [self.shares(t) for t in (r, (r >> WORD(f)) & WORD((1 << (31 - f)) - 1), r >> WORD(31))]

    def value(self, shares):
        return shares.sum(0, dtype=WORD).view(np.int32) / 2.0 ** self.f


def total(x):
    return x.sum(0, dtype=WORD)


def mask_of(x):
    return total(x[1])


# ---- attention ------------------------------------------------------------------------------------------------
F, G = 9, 6
U = 2.0 ** -F
BATCH, HEADS, TOKENS, DK, DV, CHUNK, LENGTHS = 3, 2, 10, 2, 2, 4, np.array((10, 6, 0))
CHUNKS = -(-TOKENS // CHUNK)
DECAY = np.array([[round((1 - 2.0 ** -(3 + h)) ** j * 2 ** G) for j in range(CHUNK + 1)] for h in range(HEADS)], WORD)
# Factors are at most 1/2 and off by less than u = 2^-9 from encoding, weights at most one and the table's own; truncation moves a result by at most u.
# A product of two factors is off by u + u^2.  A score: two of them and its truncation, 3.01 u, and at most 1/2.  A state: ten products, three chunks' truncations and what it began as,
# 14.02 u, and at most 10 / 4 + 1/2 = 3.  A result: four scores times values, 4 (3.01 / 2 + 1/2 + 3.01 u) u < 8.1 u; two queries times a state, 2 (14.02 / 2 + 3 + 14.02 u) u < 20.1 u;
# its truncation u: below 29.3 u.  A gradient has the same sums with the result's gradient, of the same sizes, in the place of one factor.
STATE, RESULT = 14.1 * U, 29.3 * U


class Attention:
    def __init__(self, seed):
        self.d = Dealer(seed, F)
        self.kw = dict(f=F, decay=DECAY, g=G, lengths=LENGTHS)

    def parts(self):
        for b, c, rows in lin.chunks_of(TOKENS, CHUNK, LENGTHS, BATCH):
            for h in range(HEADS):
                yield b, h, c, rows, rows.stop - rows.start, DECAY[h]

    def call(self, fn, C, f=F + G, **kw):
        return lambda *ops: fn(*ops, self.d.shares(C), self.d.tuple(C.shape, f), **self.kw, **kw)

    def scores(self, x, y):
        C = np.zeros((BATCH, HEADS, CHUNKS, CHUNK, CHUNK), WORD)
        for b, h, c, rows, L, w in self.parts():
            i, j = np.indices((L, L))
            C[b, h, c, :L, :L] = w[np.maximum(i - j, 0)] * (mask_of(x)[b, h, rows] @ mask_of(y)[b, h, rows].T)
        return self.call(lin.scores, C)(x, y)

    def states(self, x, y, first, reverse=False):
        C = np.zeros((BATCH, HEADS, CHUNKS, x[0].shape[-1], y[0].shape[-1]), WORD)
        for b, h, c, rows, L, w in self.parts():
            C[b, h, c] = (mask_of(x)[b, h, rows] * (w[1:L + 1] if reverse else w[:L][::-1])[:, None]).T @ mask_of(y)[b, h, rows]
        return self.call(lin.states, C, chunk=CHUNK, first=first, reverse=reverse)(x, y)

    def outputs(self, P, y, x, S, reverse=False, transposed=False):
        C = np.zeros((BATCH, HEADS, TOKENS, y[0].shape[-1]), WORD)
        for b, h, c, rows, L, w in self.parts():
            p, s = mask_of(P)[b, h, c, :L, :L] * np.tri(L, dtype=WORD), mask_of(S)[b, h, c]
            C[b, h, rows] = ((p.T if reverse else p) @ mask_of(y)[b, h, rows] << WORD(G)) + \
                (mask_of(x)[b, h, rows] * (w[:L][::-1] if reverse else w[1:L + 1])[:, None]) @ (s.T if transposed else s)
        return self.call(lin.outputs, C, reverse=reverse, transposed=transposed)(P, y, x, S)


def recurrence(q, k, v, first):
    """(results, last states) in float64; the decay over a whole chunk is the table's."""
    out, last = np.zeros((BATCH, HEADS, TOKENS, DV)), first.copy()
    for b, c, rows in lin.chunks_of(TOKENS, CHUNK, LENGTHS, BATCH):
        L = rows.stop - rows.start
        for h in range(HEADS if L else 0):
            w, (Q, K, V), S = DECAY[h] / 2.0 ** G, (x[b, h, rows] for x in (q, k, v)), last[b, h].copy()
            i, j = np.indices((L, L))
            out[b, h, rows] = w[1:L + 1, None] * (Q @ S) + (np.tri(L) * w[np.maximum(i - j, 0)] * (Q @ K.T)) @ V
            last[b, h] = w[L] * S + (K * w[:L][::-1, None]).T @ V
    return out, last


def test_attention_and_its_gradients():
    a, rng = Attention(11), np.random.default_rng(12)
    keys, values, state = (BATCH, HEADS, TOKENS, DK), (BATCH, HEADS, TOKENS, DV), (BATCH, HEADS, DK, DV)
    q, k, v, dO, dlast, first = (rng.uniform(-0.5, 0.5, s) for s in (keys, keys, values, values, state, state))
    Q, K, V, DO = (a.d.masked(a.d.encode(x)) for x in (q, k, v, dO))
    P = a.d.masked(a.scores(Q, K))
    states, last = a.states(K, V, a.d.encode(first))
    S = a.d.masked(states)
    out, want = a.d.value(a.outputs(P, V, Q, S)), recurrence(q, k, v, first)
    assert np.abs(out - want[0]).max() < RESULT and np.abs(a.d.value(last) - want[1]).max() < STATE
    dP = a.d.masked(a.scores(DO, V))
    back, dfirst = a.states(Q, DO, a.d.encode(dlast), reverse=True)
    dS = a.d.masked(back)
    grads = dict(q=a.outputs(dP, K, DO, S, transposed=True), k=a.outputs(dP, Q, V, dS, reverse=True, transposed=True), v=a.outputs(P, DO, K, dS, reverse=True), first=dfirst)
    point = dict(q=q, k=k, v=v, first=first)
    seen = (np.arange(TOKENS) < LENGTHS[:, None])[:, None, :, None]

    def loss(p):
        o, end = recurrence(**p)
        return (seen * o * dO).sum() + (end * dlast).sum()
    base = loss(point)
    for name, g in grads.items():
        for at in np.ndindex(point[name].shape):              # linear in each factor by itself: a step of one shows the derivative
            moved = point[name].copy()
            moved[at] += 1
            assert abs(a.d.value(g)[at] - (loss(dict(point, **{name: moved})) - base)) < (STATE if name == "first" else RESULT), (name, at)


def test_steps_are_the_recurrence():
    d, rng = Dealer(13, F), np.random.default_rng(14)
    q, k, v, first = (rng.uniform(-0.5, 0.5, s) for s in [(8, BATCH, HEADS, DK)] * 2 + [(8, BATCH, HEADS, DV), (BATCH, HEADS, DK, DV)])
    S, real, w = d.encode(first), first.copy(), DECAY[:, :2]
    lam = (w / 2.0 ** G)[None, :, :, None, None]
    for t in range(8):
        Q, K, V = (d.masked(d.encode(x[t])) for x in (q, k, v))
        mask = d.words(*S.shape)
        CS = w[None, :, 0, None, None] * mask_of(K)[..., None] * mask_of(V)[:, :, None]
        CO = (mask_of(Q)[..., None] * total(mask)).sum(-2, dtype=WORD)
        out, S = lin.step(S, Q, K, V, mask, (d.shares(CS), d.shares(CO)), (d.tuple(CS.shape, F + G), d.tuple(CO.shape, F)), F, w, G)
        real = lam[:, :, 1] * real + lam[:, :, 0] * k[t][..., None] * v[t][:, :, None]
        # a step adds u + u^2 of its product and its truncation's u to the u that the state began with: 17.1 u after eight, on states of at most 2.5; two queries times that
        # and a truncation: 2 (17.1 / 2 + 2.5 + 17.1 u) u + u < 23.3 u
        assert np.abs(d.value(S) - real).max() < 17.1 * U and np.abs(d.value(out) - (q[t][:, :, None] @ real)[:, :, 0]).max() < 23.3 * U


# ---- layer norm -----------------------------------------------------------------------------------------------
ROWS, DIM, SHIFT, ITERATIONS, EPS = 6, 8, 15, 6, 1         # 1 / dim is exact


def row_words(d, count, cuts, others):
    """[N, count, ROWS] of tuples (place -> bits) and words (place -> what it opens to)."""
    words = dict(others)
    for k, f in cuts.items():
        for j, t in enumerate(d.tuple((ROWS,), f)):
            words[k + j] = t
    return np.stack([words[k] if words[k].ndim == 2 else d.shares(words[k]) for k in range(count)], 1)


@pytest.mark.parametrize("f", [9, 12])
def test_norm_and_its_gradients(f):
    d, u, line = Dealer(15 + f, f), 2.0 ** -f, (3 << (f - 1), 1 << (f - 2))
    rng = np.random.default_rng(16)
    x = rng.uniform(-1, 1, (ROWS, DIM))
    x = (x - x.mean(-1, keepdims=True)) / x.std(-1, keepdims=True) * np.sqrt(np.linspace(0.6, 1.4, ROWS))[:, None] + rng.uniform(-1, 1, (ROWS, 1))      # variances of 0.6 to 1.4
    gamma, beta, dy = rng.uniform(0.5, 1, DIM), rng.uniform(-1, 1, DIM), rng.uniform(-1, 1, (ROWS, DIM))
    GAMMA = d.masked(d.encode(gamma))
    m1, m2, a1, a3 = (d.words(N, ROWS, DIM) for _ in range(4))
    o1, o2, p1, p3 = (total(m) for m in (m1, m2, a1, a3))
    mv, last = d.words(ROWS), d.words(ROWS)
    cuts, others = {0: SHIFT, 4: f, 7: SHIFT, 10: f}, {3: (o1 * o1).sum(-1, dtype=WORD), 13: mv}
    for k in range(14, 14 + 15 * ITERATIONS, 15):
        my, mu, mh = (d.words(ROWS) for _ in range(3))
        cuts.update({k + 2: f, k + 7: f, k + 12: f + 1})
        others.update({k: my, k + 1: my * my, k + 5: mu, k + 6: mu * mv, k + 10: mh, k + 11: my * mh})
    others[14 + 15 * ITERATIONS] = last
    # a word's mask is shared once: what is opened and what is multiplied are the same shares
    words = row_words(d, 15 * (ITERATIONS + 1), cuts, others)
    cut = d.tuple((ROWS, DIM), f), d.tuple((ROWS, DIM), f)
    out, xhat, rstd = lin.layernorm(d.encode(x), GAMMA, d.encode(beta), (m1, m2), (d.shares(o1 * last[:, None]), d.shares(o2 * mask_of(GAMMA))), cut, words, f, SHIFT, line, EPS)

    def norm(x, gamma, beta):
        c = x - x.mean(-1, keepdims=True)
        r = 1 / np.sqrt((c * c).mean(-1, keepdims=True) + EPS * u)
        return c * r * gamma + beta, c * r, r[:, 0]
    want = norm(x, gamma, beta)
    # Encoding moves a value up to u down, so a mean by that and its truncation's u: centred words are off by less than 2 u.  The variance: 2 |c| 2 u + 4 u^2 a term, of |c| whose mean is
    # at most its root; the truncation of the sum, u / 8, and of the mean, u.  1 / sqrt(v) by half of v^(-3/2) of that.  A Newton step by its own roundings: y (v u + u) / 2 + u, 2.1 u here;
    # six are enough for both ends of the variances to converge, and what is left of the step before counts squared, less than 0.1 u.
    A, X, R = np.abs(x - x.mean(-1, keepdims=True)).max(), np.abs(want[1]).max(), want[2].max()
    e_v = 4 * 1.4 ** 0.5 * u + 4 * u * u + 1.125 * u
    e_r = 0.5 * (0.6 - e_v) ** -1.5 * e_v + 2.2 * u
    e_x = 2 * u * R + A * e_r + 2 * u * e_r + u
    assert np.abs(d.value(rstd) - want[2]).max() < e_r and np.abs(d.value(xhat) - want[1]).max() < e_x
    assert np.abs(d.value(out) - want[0]).max() < e_x * (1 + u) + X * u + 2 * u
    # backward
    ma, mb, mk = (d.words(ROWS) for _ in range(3))
    words = row_words(d, 22, {0: SHIFT, 4: f, 7: SHIFT, 13: f, 18: f},
                      {3: (p3 * o2).sum(-1, dtype=WORD), 10: last, 11: ma, 12: ma * last, 16: mb, 17: mb * last, 21: mk})
    columns = np.stack([d.shares((p1 * o2).sum(0, dtype=WORD))] + d.tuple((DIM,), f), 1)
    dx, dgamma, dbeta = lin.layernorm_grad(d.encode(dy), xhat, rstd, GAMMA, (a1, m2, a3), (d.shares(p1 * mask_of(GAMMA)), d.shares(p3 * last[:, None] - o2 * mk[:, None])),
                                           (d.tuple((ROWS, DIM), f), d.tuple((ROWS, DIM), f)), words, columns, f, SHIFT)
    # dy, gamma and g = dy gamma are at most one; g is off by 2 u + u^2 and its truncation's u; the means by their terms, with truncations of u and 1.125 u; k1 and k2 are their products
    # with rstd, dx two products of three terms
    e_g = 3 * u + u * u
    e_m1, e_m2 = e_g + u, e_x + X * e_g + e_x * e_g + 1.125 * u
    e_k1, e_k2 = e_r + R * e_m1 + e_r * e_m1 + u, X * e_r + R * e_m2 + e_r * e_m2 + u       # |m1| at most 1, |m2| at most X
    bounds = dict(x=e_r + R * e_g + e_r * e_g + X * e_k2 + X * R * e_x + e_x * e_k2 + u + e_k1, gamma=ROWS * (e_x * (1 + u) + X * u) + u, beta=ROWS * u)
    point, h = dict(x=x, gamma=gamma, beta=beta), 1e-5        # central differences: their own error is below 1e-7 here

    def loss(**p):
        return (norm(**p)[0] * dy).sum()
    for name, got in (("x", dx), ("gamma", dgamma), ("beta", dbeta)):
        for at in np.ndindex(point[name].shape):
            up, down = point[name].copy(), point[name].copy()
            up[at] += h
            down[at] -= h
            slope = (loss(**dict(point, **{name: up})) - loss(**dict(point, **{name: down}))) / (2 * h)
            assert abs(d.value(got)[at] - slope) < bounds[name] + 1e-7, (name, at)
