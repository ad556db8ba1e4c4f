"""What pins the numpy oracle of the cache, its attention and the bias: a cached row reconstructs, products reconstruct to the plain product of what the
tree sees, the gradient is the difference quotient (the bias is linear, so exactly), buckets follow the logarithm."""
import math

import numpy as np
import pytest

import oracle
from oracle import generation as gen
from paper_2402_02320_amd import spin


def uniform(rng, dtype, *shape):
    return rng.integers(0, 1 << 8 * np.dtype(dtype).itemsize, size=shape, dtype=np.uint64 if dtype == np.uint64 else np.int64).astype(dtype)


def share(rng, x, n):
    parts = uniform(rng, x.dtype, n, *x.shape)
    parts[0] = x - parts[1:].sum(0, dtype=x.dtype)
    return parts


@pytest.mark.parametrize("dtype", [np.uint64, np.uint32])
@pytest.mark.parametrize("n", [1, 2, 3])
def test_attention_reconstructs(dtype, n):
    rng = np.random.default_rng(n)
    batch, heads, cached, nodes, dim, tokens, context = 2, 4, 2, 3, 8, 16, np.array([19, 0])
    table = np.array([[3, 0], [1, 4]], np.int32)
    pool = uniform(rng, dtype, n + 1, 6, cached, tokens, dim)
    columns = 22
    k = uniform(rng, dtype, batch, cached, columns, dim)
    mask = uniform(rng, dtype, n, batch, cached, columns, dim)
    pool = gen.append(pool, table, np.zeros(batch, int), None, share(rng, k, n), mask)
    for b in range(batch):
        for g in range(cached):
            rows = gen.cached_rows(pool, table, b, g, columns)
            assert (rows[1:].sum(0, dtype=dtype) == k[b, g]).all()                       # slots 1 to n are a sharing of the row
            assert (rows[0] == k[b, g] - mask[:, b, g].sum(0, dtype=dtype)).all()        # slot 0 is public
    tree = np.array([[1, 3, 5], [1, 2, 6]])
    seen = gen.visible(pool, table, context, tree, nodes, columns)
    q = uniform(rng, dtype, batch, heads, nodes, dim)
    A = uniform(rng, dtype, n, batch, heads, nodes, dim)
    a, m = A.sum(0, dtype=dtype), mask.sum(0, dtype=dtype)
    C = share(rng, np.stack([np.stack([a[b, h] @ m[b, h // 2].T for h in range(heads)]) for b in range(batch)]), n)
    got = gen.scores(pool, table, context, share(rng, q, n), A, C, tree=tree, masked=7).sum(0, dtype=dtype)
    for b in range(batch):
        for h in range(heads):
            assert (got[b, h] == np.where(seen[b], q[b, h] @ k[b, h // 2].T, dtype(7))).all()
    p = uniform(rng, dtype, batch, heads, nodes, columns)
    A = uniform(rng, dtype, n, batch, heads, nodes, columns)
    a = np.where(seen[:, None], A.sum(0, dtype=dtype), dtype(0))
    C = share(rng, np.stack([np.stack([a[b, h] @ m[b, h // 2] for h in range(heads)]) for b in range(batch)]), n)
    got = gen.values(pool, table, context, share(rng, p, n), A, C, tree=tree).sum(0, dtype=dtype)
    for b in range(batch):
        for h in range(heads):
            assert (got[b, h] == np.where(seen[b], p[b, h], dtype(0)) @ k[b, h // 2]).all()


def test_truncation_of_both_rings_is_the_oracles():
    rng = np.random.default_rng(1)
    for dtype, bits in ((np.uint64, 64), (np.uint32, 32)):
        x = rng.integers(-1 << bits - 3, 1 << bits - 3, size=100)
        r = uniform(rng, dtype, 100)
        tup = [share(rng, t.astype(dtype), 3) for t in (r, (r >> dtype(9)) & dtype((1 << bits - 10) - 1), r >> dtype(bits - 1))]
        got = gen.trunc(share(rng, x.astype(dtype), 3), tup, 9).sum(0, dtype=dtype).astype(f"int{bits}")
        assert set((got.astype(np.int64) - (x >> 9)).tolist()) <= {0, 1}


@pytest.mark.parametrize("causal,lengths,first", [(False, None, 0), (True, [5, 3], 0), (True, [9, 1], 4), (True, [9, 9], -2)])
def test_gradient_is_the_difference(causal, lengths, first):
    rng = np.random.default_rng(3)
    n, batch, heads, Q, K, buckets, reach = 2, 2, 3, 6, 9, 6, 8
    lut = spin.relative_buckets(buckets, reach, not causal).numpy()
    x, w = uniform(rng, np.uint64, n, batch, heads, Q, K), uniform(rng, np.uint64, n, batch, heads, Q, K)
    table = uniform(rng, np.uint64, n, heads, buckets)
    kw = dict(first=first, causal=causal, lengths=lengths)
    grad = gen.relbias_grad(w, lut, buckets, **kw)
    base = gen.relbias_trunc(x, table, lut, **kw)
    for h in range(heads):
        for k in range(buckets):
            more = table.copy()
            more[:, h, k] += np.uint64(1)
            d = gen.relbias_trunc(x, more, lut, **kw) - base
            assert ((w * d).sum((1, 2, 3, 4), dtype=np.uint64) == grad[:, h, k]).all()


@pytest.mark.parametrize("buckets,reach,both", [(32, 128, True), (32, 128, False), (8, 20, True), (4, 3, False), (64, 4000, False)])
def test_buckets(buckets, reach, both):
    lut = spin.relative_buckets(buckets, reach, both).tolist()
    half = buckets // 2 if both else buckets
    near = half // 2
    for d in range(-reach, reach + 1):
        m = abs(d) if both else max(-d, 0)
        got = lut[d + reach] - (half if both and d > 0 else 0)
        want = near + math.log(max(m, near) / near) / math.log(reach / near) * (half - near)
        if m < near:
            assert got == m
        else:                                                # within rounding of a border either side is the logarithm's
            assert min(int(want - 1e-9), half - 1) <= got <= min(int(want + 1e-9), half - 1)
    assert lut[0] == half - 1
    for bad in ((1, 10, False), (8, 2, False), (7, 20, True), (2, 20, True)):
        with pytest.raises(spin.SpinError):
            spin.relative_buckets(*bad)
