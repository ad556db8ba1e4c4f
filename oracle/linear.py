"""Linear attention with a decay and layer norm on shares, word by word in numpy (test infrastructure only).

Written from the definitions in include/spin.h; unsigned numpy integers wrap as the ring does.  All arrays are on the host; ring arrays are numpy
uint64 or uint32.  A factor is a pair (shares, masks), party axis first."""
import numpy as np

from oracle.generation import trunc


def opened(x):
    value, mask = x
    return value.sum(0, dtype=value.dtype) - mask.sum(0, dtype=mask.dtype)


def beaver(x, y, times):
    """[n] + ...: every party's part of x . y, by the bilinear `times`."""
    e, f = opened(x), opened(y)
    z = np.stack([times(x[1][i], f) + times(e, y[1][i]) for i in range(len(x[0]))])
    z[0] += times(e, f)
    return z


def weights(decay, head, chunk, dtype):
    return np.ones(chunk + 1, dtype) if decay is None else decay[head]


def chunks_of(tokens, chunk, lengths, batch):
    """(sequence, chunk, its tokens that are there) of all."""
    for b in range(batch):
        length = tokens if lengths is None else min(max(int(lengths[b]), 0), tokens)
        for c in range(-(-tokens // chunk)):
            yield b, c, slice(c * chunk, max(c * chunk, min((c + 1) * chunk, length)))


def rows_of(x, b, h, rows):
    return tuple(v[:, b, h, rows] for v in x)


def turned(x):
    return tuple(v.swapaxes(-1, -2) for v in x)


def weighed(x, w):
    return tuple(v * w[:, None] for v in x)


def scores(x, y, C, t, f, decay=None, g=0, lengths=None):
    out = np.zeros_like(C)
    n, batch, heads, tokens, _ = x[0].shape
    chunk = C.shape[-1]
    for b, c, rows in chunks_of(tokens, chunk, lengths, batch):
        L = rows.stop - rows.start
        for h in range(heads if L else 0):
            w = weights(decay, h, chunk, C.dtype)
            z = beaver(rows_of(x, b, h, rows), turned(rows_of(y, b, h, rows)), np.matmul)
            at = (slice(None), b, h, c, slice(0, L), slice(0, L))
            i, j = np.indices((L, L))
            z = trunc(C[at] + w[np.maximum(i - j, 0)] * z, [v[at] for v in t], f + g)
            out[at] = np.where(j <= i, z, C.dtype.type(0))
    return out


def states(x, y, C, t, f, chunk, decay=None, g=0, lengths=None, first=None, reverse=False):
    n, batch, heads, tokens, rows_ = x[0].shape
    out, last = np.zeros_like(C), np.zeros(C.shape[:3] + C.shape[4:], C.dtype) if first is None else first.copy()
    order = list(chunks_of(tokens, chunk, lengths, batch))
    for b, c, rows in order[::-1] if reverse else order:
        L = rows.stop - rows.start
        for h in range(heads):
            out[:, b, h, c] = last[:, b, h]
            if L:
                w = weights(decay, h, chunk, C.dtype)
                left = turned(weighed(rows_of(x, b, h, rows), w[1:L + 1] if reverse else w[:L][::-1]))
                z = beaver(left, rows_of(y, b, h, rows), np.matmul) + C[:, b, h, c] + (w[L] << C.dtype.type(f)) * last[:, b, h]
                last[:, b, h] = trunc(z, [v[:, b, h, c] for v in t], f + g)
    return out, last


def outputs(P, y, x, S, C, t, f, decay=None, g=0, lengths=None, reverse=False, transposed=False):
    out = np.zeros_like(C)
    n, batch, heads, tokens, _ = x[0].shape
    chunk = P[0].shape[-1]
    for b, c, rows in chunks_of(tokens, chunk, lengths, batch):
        L = rows.stop - rows.start
        for h in range(heads if L else 0):
            w = weights(decay, h, chunk, C.dtype)
            p = tuple(v[:, b, h, c, :L, :L] * np.tri(L, dtype=C.dtype) for v in P)
            s = tuple(v[:, b, h, c] for v in S)
            z = beaver(turned(p) if reverse else p, rows_of(y, b, h, rows), np.matmul) << C.dtype.type(g)
            z = z + beaver(weighed(rows_of(x, b, h, rows), w[:L][::-1] if reverse else w[1:L + 1]), turned(s) if transposed else s, np.matmul)
            out[:, b, h, rows] = trunc(z + C[:, b, h, rows], [v[:, b, h, rows] for v in t], f + g)
    return out


def step(S, q, k, v, mask, C, tuples, f, decay=None, g=0, active=None):
    out, after = np.zeros_like(C[1]), S.copy()
    for b in range(S.shape[1]):
        if active is not None and active[b] <= 0:
            continue
        for h in range(S.shape[2]):
            w = weights(decay, h, 1, S.dtype)
            column, row, query = (tuple(t[:, b, h, :, None] for t in k), tuple(t[:, b, h, None] for t in v), tuple(t[:, b, h, None] for t in q))
            z = C[0][:, b, h] + (w[1] << S.dtype.type(f)) * S[:, b, h] + w[0] * beaver(column, row, np.matmul)
            after[:, b, h] = trunc(z, [t[:, b, h] for t in tuples[0]], f + g)
            z = C[1][:, b, h] + beaver(query, (after[:, b, h], mask[:, b, h]), np.matmul)[:, 0]
            out[:, b, h] = trunc(z, [t[:, b, h] for t in tuples[1]], f)
    return out, after


def _words(w):
    """word(k), cut(y, k, bits) of [n, words, ..]"""
    return (lambda k: w[:, k]), (lambda y, k, bits: trunc(np.ascontiguousarray(y), [np.ascontiguousarray(w[:, k + j]) for j in range(3)], bits))


def _public(y, v):
    y = y.copy()
    y[0] += y.dtype.type(v % (1 << 8 * y.dtype.itemsize))
    return y


def _tall(v, dim):
    return np.repeat(v[..., None], dim, -1)


def inverse(shift, dim, dtype):
    return dtype.type(((1 << shift) + dim // 2) // dim)


def layernorm(x, gamma, beta, masks, C, tuples, row_words, f, shift, line, eps=0):
    n, rows, dim = x.shape
    word, cut = _words(row_words)
    inv, slope = inverse(shift, dim, x.dtype), x.dtype.type(line[1] % (1 << 8 * x.dtype.itemsize))
    centred = x - _tall(cut(x.sum(-1, dtype=x.dtype) * inv, 0, shift), dim)
    square = beaver((centred, masks[0]), (centred, masks[0]), np.multiply).sum(-1, dtype=x.dtype) + word(3)
    v = _public(cut(cut(square, 4, f) * inv, 7, shift), eps)
    y = cut(_public(x.dtype.type(0) - slope * v, line[0] << f), 10, f)
    for k in range(14, row_words.shape[1] - 1, 15):
        u = cut(word(k + 1) + beaver((y, word(k)), (y, word(k)), np.multiply), k + 2, f)
        h = cut(word(k + 6) + beaver((u, word(k + 5)), (v, word(13)), np.multiply), k + 7, f)
        h = _public(x.dtype.type(0) - h, 3 << f)
        y = cut(word(k + 11) + beaver((y, word(k)), (h, word(k + 10)), np.multiply), k + 12, f + 1)
    b = word(row_words.shape[1] - 1)
    xhat = trunc(C[0] + beaver((centred, masks[0]), (_tall(y, dim), _tall(b, dim)), np.multiply), tuples[0], f)
    wide = tuple(np.repeat(v[:, None], rows, 1) for v in gamma)
    return trunc(C[1] + beaver((xhat, masks[1]), wide, np.multiply), tuples[1], f) + beta[:, None], xhat, y


def layernorm_grad(dy, xhat, rstd, gamma, masks, C, tuples, row_words, column_words, f, shift):
    n, rows, dim = dy.shape
    word, cut = _words(row_words)
    column, cut_column = _words(column_words)
    inv = inverse(shift, dim, dy.dtype)
    wide = tuple(np.repeat(v[:, None], rows, 1) for v in gamma)
    g = trunc(C[0] + beaver((dy, masks[0]), wide, np.multiply), tuples[0], f)
    dgamma = cut_column(column(0) + beaver((dy, masks[0]), (xhat, masks[1]), np.multiply).sum(1, dtype=dy.dtype), 1, f)
    m1 = cut(g.sum(-1, dtype=dy.dtype) * inv, 0, shift)
    m2 = cut(cut(word(3) + beaver((g, masks[2]), (xhat, masks[1]), np.multiply).sum(-1, dtype=dy.dtype), 4, f) * inv, 7, shift)
    r = (rstd, word(10))
    k1 = cut(word(12) + beaver((m1, word(11)), r, np.multiply), 13, f)
    k2 = cut(word(17) + beaver((m2, word(16)), r, np.multiply), 18, f)
    z = C[1] + beaver((g, masks[2]), tuple(_tall(v, dim) for v in r), np.multiply)
    z = z - beaver((xhat, masks[1]), (_tall(k2, dim), _tall(word(21), dim)), np.multiply)
    return trunc(z, tuples[1], f) - _tall(k1, dim), dgamma, dy.sum(1, dtype=dy.dtype)
