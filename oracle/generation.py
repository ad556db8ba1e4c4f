"""The paged cache of shares, attention over it and the relative position bias, word by word in numpy (test infrastructure only).

Written from the definitions in include/spin.h; unsigned numpy integers wrap as the ring does.  All arrays are on the host; ring arrays are numpy
uint64 or uint32.  Truncation is the C oracle's."""
import numpy as np

import oracle


def trunc(y, tup, f):
    if not f:
        return y
    n = y.shape[0]
    bits = 8 * y.dtype.itemsize
    wide = [np.ascontiguousarray(t.reshape(n, -1).astype(np.uint64)) for t in (y,) + tuple(tup)]
    return oracle.trunc(*wide, f, l=bits).astype(y.dtype).reshape(y.shape)


def place(pool, table, b, pos):
    """(page, place in the page) of a position, or None."""
    tokens = pool.shape[3]
    if pos < 0 or pos // tokens >= table.shape[1]:
        return None
    page = int(table[b, pos // tokens])
    return (page, pos % tokens) if 0 <= page < pool.shape[1] else None


def append(pool, table, start, count, x, mask):
    """The pool afterwards.  x, mask: [n, batch, heads, rows, dim]."""
    pool = pool.copy()
    for b in range(x.shape[1]):
        for s in range(x.shape[3] if count is None else min(int(count[b]), x.shape[3])):
            at = place(pool, table, b, int(start[b]) + s)
            if at is None:
                continue
            opened = (x[:, b, :, s] - mask[:, b, :, s]).sum(0, dtype=x.dtype)
            pool[0, at[0], :, at[1]] = opened
            pool[1:, at[0], :, at[1]] = mask[:, b, :, s]
            pool[1, at[0], :, at[1]] += opened
    return pool


def copy(pool, src, dst):
    pool = pool.copy()
    for s, d in zip(src, dst):
        if 0 <= s < pool.shape[1] and 0 <= d < pool.shape[1]:
            pool[:, d] = pool[:, s]
    return pool


def compact(pool, table, context, kept, kept_count):
    old, pool = pool, pool.copy()
    for b in range(kept.shape[0]):
        for j in range(min(int(kept_count[b]), kept.shape[1])):
            if context[b] < 0 or not 0 <= kept[b, j] < kept.shape[1]:
                continue
            at, to = place(old, table, b, int(context[b]) + int(kept[b, j])), place(old, table, b, int(context[b]) + j)
            if at is not None and to is not None:
                pool[:, to[0], :, to[1]] = old[:, at[0], :, at[1]]
    return pool


def visible(pool, table, context, tree, nodes, columns):
    """[batch, nodes, columns]"""
    seen = np.zeros((table.shape[0], nodes, columns), bool)
    for b in range(table.shape[0]):
        for t in range(columns if context[b] >= 0 else 0):
            j = t - int(context[b])
            if j >= nodes or place(pool, table, b, t) is None:
                continue
            for m in range(nodes):
                seen[b, m, t] = j < 0 or (int(tree[b, m]) >> j & 1 if tree is not None else j <= m)
    return seen


def cached_rows(pool, table, b, head, columns):
    """[slots, columns, dim], zero where there is no page."""
    out = np.zeros((pool.shape[0], columns, pool.shape[4]), pool.dtype)
    for t in range(columns):
        at = place(pool, table, b, t)
        if at is not None:
            out[:, t] = pool[:, at[0], head, at[1]]
    return out


def bias_of(table, bucket_of, head, distance):
    """[n] + distance.shape"""
    reach = len(bucket_of) // 2
    bucket = bucket_of[np.clip(distance, -reach, reach) + reach]
    ok = (bucket >= 0) & (bucket < table.shape[2])
    return np.where(ok, table[:, head][:, np.where(ok, bucket, 0)], np.array(0, table.dtype))


def scores(pool, table, context, Q, A, C, f=0, tup=None, tree=None, masked=0, bias=None, depth=None):
    n, batch, heads, nodes, _ = Q.shape
    columns = C.shape[4]
    seen = visible(pool, table, context, tree, nodes, columns)
    z = C.copy()
    for b in range(batch):
        for h in range(heads):
            rows = cached_rows(pool, table, b, h // (heads // pool.shape[2]), columns)
            e = (Q[:, b, h] - A[:, b, h]).sum(0, dtype=Q.dtype)
            for i in range(n):
                z[i, b, h] += e @ rows[1 + i].T + A[i, b, h] @ rows[0].T
    z = trunc(z, tup, f)
    for b in range(batch):
        at = np.arange(nodes) if depth is None else depth[b].astype(np.int64)
        keys = np.arange(columns) - int(context[b])
        keys[(keys >= 0) & (keys < nodes)] = at[keys[(keys >= 0) & (keys < nodes)]]
        for h in range(heads):
            if bias is not None:
                z[:, b, h] += bias_of(bias[0], bias[1], h, keys[None, :] - at[:, None])
            for i in range(n):
                z[i, b, h] = np.where(seen[b], z[i, b, h], z.dtype.type(masked if i == 0 else 0))
    return z


def values(pool, table, context, P, A, C, f=0, tup=None, tree=None):
    n, batch, heads, nodes, columns = P.shape
    seen = visible(pool, table, context, tree, nodes, columns)
    z = C.copy()
    for b in range(batch):
        for h in range(heads):
            rows = cached_rows(pool, table, b, h // (heads // pool.shape[2]), columns)
            e = np.where(seen[b], (P[:, b, h] - A[:, b, h]).sum(0, dtype=P.dtype), P.dtype.type(0))
            for i in range(n):
                z[i, b, h] += e @ rows[1 + i] + np.where(seen[b], A[i, b, h], P.dtype.type(0)) @ rows[0]
    return trunc(z, tup, f)


def pairs(batch, Q, K, first, causal, lengths):
    seen = np.ones((batch, Q, K), bool)
    if lengths is not None:
        seen &= np.arange(K) < np.asarray(lengths)[:, None, None]
    if causal:
        seen &= np.arange(K) <= np.arange(Q)[:, None] + first
    return seen


def relbias_trunc(x, table, bucket_of, f=0, tup=None, first=0, causal=False, lengths=None, masked=0):
    n, batch, heads, Q, K = x.shape
    seen, away = pairs(batch, Q, K, first, causal, lengths), np.arange(K) - np.arange(Q)[:, None] - first
    y = trunc(x, tup, f).copy()
    for h in range(heads):
        y[:, :, h] += bias_of(table, bucket_of, h, away)[:, None]
    for i in range(n):
        y[i] = np.where(seen[:, None], y[i], y.dtype.type(masked if i == 0 else 0))
    return y


def relbias_grad(dS, bucket_of, buckets, first=0, causal=False, lengths=None):
    n, batch, heads, Q, K = dS.shape
    reach = len(bucket_of) // 2
    bucket = bucket_of[np.clip(np.arange(K) - np.arange(Q)[:, None] - first, -reach, reach) + reach]
    seen = pairs(batch, Q, K, first, causal, lengths)
    out = np.zeros((n, heads, buckets), dS.dtype)
    for k in range(buckets):
        there = (seen & (bucket == k))[:, None]
        out[:, :, k] = np.where(there, dS, dS.dtype.type(0)).sum((1, 3, 4), dtype=dS.dtype)
    return out
