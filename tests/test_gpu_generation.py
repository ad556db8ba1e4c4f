"""The paged cache of shares, attention of new tokens over it and the relative position bias, word for word against the numpy oracle: both rings, one to
eight parties, shared heads, ragged and empty contexts, trees, pages that are not there, other streams, graphs, offsets past 32 bits."""
import numpy as np
import pytest
import torch

from oracle import generation as gen
from paper_2402_02320_amd import spin

pytestmark = pytest.mark.gpu

RINGS = {64: (spin, np.uint64, np.int64), 32: (spin.ring32, np.uint32, np.int32)}
BITS = pytest.mark.parametrize("bits", [64, 32])


def uniform(rng, bits, *shape):
    return rng.integers(0, 1 << bits, size=shape, dtype=np.uint64).astype(RINGS[bits][1])


def dev(a):
    a = np.ascontiguousarray(a)
    return torch.from_numpy(a.view({8: np.int64, 4: np.int32}[a.dtype.itemsize])).cuda()


def ints(a):
    return torch.tensor(np.asarray(a), dtype=torch.int32, device="cuda")


def same(got, want):
    return np.array_equal(got.cpu().numpy().view(want.dtype), want)


def table_of(rng, batch, table_pages, pages):
    return rng.permutation(pages)[:batch * table_pages].reshape(batch, table_pages).astype(np.int32)


def tuple_of(rng, bits, shape):
    return [uniform(rng, bits, *shape) for _ in range(3)]


def random_tree(rng, batch, nodes):
    tree = rng.integers(0, 1 << nodes, size=(batch, nodes), dtype=np.uint64) if nodes < 64 else rng.integers(0, 1 << 63, size=(batch, nodes), dtype=np.uint64) * 2 + 1
    tree[0, 0] = 0                                            # a node that sees none of the drafted
    return tree.view(np.int64)


# name: n, batch, query heads, cached heads, nodes, dim, page tokens, contexts, columns beyond the last token, f, tree, bias, depth, bad pages
ATTENTION = {
    "token": (3, 2, 4, 4, 1, 64, 16, (40, 0), 0, 9, False, False, False, False),
    "one_of_everything": (1, 1, 1, 1, 1, 8, 16, (0,), 0, 0, False, False, False, False),
    "idle": (2, 3, 2, 1, 2, 16, 16, (-1, 5, -7), 3, 9, True, True, True, False),
    "empty_rows": (2, 2, 4, 2, 5, 24, 16, (0, 1), 1, 9, True, False, False, False),
    "chain_over_a_page": (3, 2, 6, 2, 3, 72, 16, (14, 15), 0, 9, False, True, False, False),
    "page_ends_inside": (3, 3, 8, 2, 7, 128, 32, (31, 32, 95), 5, 12, True, True, True, False),
    "rows_over_a_tile": (2, 2, 20, 4, 7, 80, 64, (65, 130), 0, 12, True, True, True, False),
    "many_nodes": (2, 1, 4, 2, 64, 40, 16, (77,), 0, 9, True, False, False, False),
    "dim_256": (3, 1, 4, 2, 2, 256, 64, (100,), 0, 9, True, True, True, False),
    "dim_200": (5, 1, 2, 1, 3, 200, 16, (50,), 0, 0, True, False, False, False),
    "four_parties": (4, 2, 4, 2, 9, 96, 16, (64, 63), 0, 9, True, True, True, False),
    "five_parties": (5, 2, 4, 4, 2, 128, 16, (17, 90), 0, 9, True, True, True, False),
    "seven_parties": (7, 1, 3, 1, 2, 32, 16, (70,), 0, 9, True, False, False, False),
    "eight_parties": (8, 2, 2, 2, 3, 128, 64, (129, 3), 2, 9, True, True, True, False),
    "eight_parties_256": (8, 1, 2, 1, 1, 256, 16, (33,), 0, 9, False, False, False, False),
    "bad_pages": (2, 3, 4, 2, 4, 64, 16, (60, 40, 100), 0, 9, True, True, True, True),
    "table_too_short": (2, 1, 2, 1, 3, 32, 16, (30,), 40, 9, True, False, False, False),
    "context_past_the_columns": (2, 2, 2, 1, 3, 32, 16, (90, 47), -40, 9, True, True, True, False),
    "longer": (3, 2, 8, 2, 3, 64, 16, (1500, 700), 0, 16, True, True, True, False),
    "long_one_head": (2, 1, 1, 1, 1, 128, 64, (9001,), 0, 16, False, False, False, False),
}


def attention_case(name, bits, seed=0):
    n, batch, heads, cached, nodes, dim, tokens, contexts, more, f, tree, bias, depth, bad = ATTENTION[name]
    rng = np.random.default_rng(seed + sum(map(ord, name)))
    columns = max(contexts) + nodes + more
    table_pages = 2 if name == "table_too_short" else -(-max(max(contexts) + nodes, 1) // tokens)
    pages = batch * table_pages + 2
    table = table_of(rng, batch, table_pages, pages)
    if bad:
        table[0, 1], table[1, 0], table[2, 2], table[2, 3] = pages, -1, 2 ** 31 - 1, -2 ** 31
    rows = (n, batch, heads, nodes)
    c = dict(n=n, f=f, columns=columns, dim=dim, rows=rows, table=table, context=np.array(contexts), pool=uniform(rng, bits, n + 1, pages, cached, tokens, dim),
             tree=random_tree(rng, batch, nodes) if tree else None, rng=rng)
    c["bias"] = None
    if bias:
        lut = spin.relative_buckets(32, 20, False).numpy().copy()
        lut[3], lut[30] = -1, 32                              # distances without a bucket
        c["bias"] = (uniform(rng, bits, n, heads, 32), lut)
    c["depth"] = rng.integers(0, 5, size=(batch, nodes)).astype(np.int32) if depth else None
    return c


def run_scores(c, bits, out=None):
    ring, rng = RINGS[bits][0], c["rng"]
    wide = c["rows"] + (c["columns"],)
    Q, A = uniform(rng, bits, *c["rows"], c["dim"]), uniform(rng, bits, *c["rows"], c["dim"])
    C, tup = uniform(rng, bits, *wide), tuple_of(rng, bits, wide) if c["f"] else None
    masked = -12345
    want = gen.scores(c["pool"], c["table"], c["context"], Q, A, C, c["f"], tup, c["tree"], masked % (1 << bits), c["bias"], c["depth"])
    Cd = dev(C)

    def call(out=None):
        return ring.cache_scores(dev(c["pool"]), ints(c["table"]), ints(c["context"]), dev(Q), dev(A), Cd, f=c["f"], tuple_=tup and [dev(t) for t in tup],
                                 tree=None if c["tree"] is None else dev(c["tree"]), masked=masked, bias=c["bias"] and (dev(c["bias"][0]), ints(c["bias"][1])),
                                 depth=None if c["depth"] is None else ints(c["depth"]), out=out)
    return call, want, Cd


def run_values(c, bits):
    ring, rng = RINGS[bits][0], c["rng"]
    P, A = uniform(rng, bits, *c["rows"], c["columns"]), uniform(rng, bits, *c["rows"], c["columns"])
    wide = c["rows"] + (c["dim"],)
    C, tup = uniform(rng, bits, *wide), tuple_of(rng, bits, wide) if c["f"] else None
    want = gen.values(c["pool"], c["table"], c["context"], P, A, C, c["f"], tup, c["tree"])

    def call(out=None, workspace=None):
        return ring.cache_values(dev(c["pool"]), ints(c["table"]), ints(c["context"]), dev(P), dev(A), dev(C), f=c["f"], tuple_=tup and [dev(t) for t in tup],
                                 tree=None if c["tree"] is None else dev(c["tree"]), out=out, workspace=workspace)
    return call, want


@BITS
@pytest.mark.parametrize("name", sorted(ATTENTION))
def test_scores(name, bits):
    call, want, C = run_scores(attention_case(name, bits), bits)
    assert same(call(), want)
    assert same(call(out=C), want)                            # in place of the triple's C


@BITS
@pytest.mark.parametrize("name", sorted(ATTENTION))
def test_values(name, bits):
    call, want = run_values(attention_case(name, bits), bits)
    assert same(call(), want)
    size = RINGS[bits][0].cache_values_workspace_bytes
    c = attention_case(name, bits)
    need = size(dev(c["pool"]), ints(c["table"]), c["rows"][2], c["rows"][3], c["columns"])
    ws = torch.full((need + 512,), 0x5A, dtype=torch.uint8, device="cuda")
    assert same(call(workspace=ws[:need]), want) and bool((ws[need:] == 0x5A).all())     # any workspace contents, no byte past its end


@BITS
@pytest.mark.parametrize("n", range(1, 9))
@pytest.mark.parametrize("rows,dim,tokens,starts,counts", [(1, 64, 16, (0, 37), None), (5, 8, 16, (14, 3), (5, 0)), (70, 128, 32, (0, 60), (70, 33)),
                                                           (33, 72, 16, (-2, 40), (33, 99))])
def test_append(bits, n, rows, dim, tokens, starts, counts):
    ring = RINGS[bits][0]
    rng = np.random.default_rng(n * 100 + rows)
    batch, heads, table_pages = 2, 3, -(-(60 + 70) // tokens)
    pages = batch * table_pages + 1
    table = table_of(rng, batch, table_pages, pages)
    table[1, 3 % table_pages] = pages + 5                     # its rows are left out
    pools = [uniform(rng, bits, n + 1, pages, heads, tokens, dim) for _ in range(2)]
    x, b = ([uniform(rng, bits, n, batch, heads, rows, dim) for _ in range(2)] for _ in range(2))
    want = [gen.append(p, table, starts, counts, x[k], b[k]) for k, p in enumerate(pools)]
    got = ring.cache_append([dev(p) for p in pools], ints(table), ints(starts), [dev(t) for t in x], [dev(t) for t in b], count=None if counts is None else ints(counts))
    assert same(got[0], want[0]) and same(got[1], want[1])


@BITS
@pytest.mark.parametrize("n,heads,tokens,dim", [(1, 1, 16, 8), (3, 5, 16, 72), (2, 8, 64, 128)])
def test_copy(bits, n, heads, tokens, dim):
    rng = np.random.default_rng(n)
    pools = [uniform(rng, bits, n + 1, 9, heads, tokens, dim) for _ in range(2)]
    src, dst = [3, 0, 3, 9, 1, -1], [4, 8, 5, 6, 1000, 7]
    got = RINGS[bits][0].cache_copy([dev(p) for p in pools], ints(src), ints(dst))
    for g, p in zip(got, pools):
        assert same(g, gen.copy(p, src, dst))


@BITS
@pytest.mark.parametrize("nodes,tokens,contexts", [(1, 16, (5, 0, 15)), (9, 16, (0, 12, -1)), (40, 16, (7, 16, 3)), (64, 32, (31, 0, 100))])
def test_compact(bits, nodes, tokens, contexts):
    rng = np.random.default_rng(nodes)
    n, heads, dim = 3, 2, 72
    table_pages = -(-(max(contexts) + nodes) // tokens)
    pages = 3 * table_pages + 2
    table = table_of(rng, 3, table_pages, pages)
    table[2, -1] = -5
    kept = np.zeros((3, nodes), np.int32)
    counts = [nodes, min(3, nodes), nodes // 2]
    for b in range(3):
        kept[b, :counts[b]] = np.sort(rng.permutation(nodes)[:counts[b]])
    if nodes > 8:
        kept[0, nodes - 2:] = nodes, 2 ** 31 - 1              # left out
        counts[1] = 2 ** 31 - 1                               # no more than the list holds
        kept[1] = np.arange(nodes)
    pools = [uniform(rng, bits, n + 1, pages, heads, tokens, dim) for _ in range(2)]
    got = RINGS[bits][0].cache_compact([dev(p) for p in pools], ints(table), ints(contexts), ints(kept), ints(counts))
    for g, p in zip(got, pools):
        assert same(g, gen.compact(p, table, contexts, kept, counts))


# n, batch, heads, Q, K, first, causal, lengths
PAIRS = [(1, 1, 1, 1, 1, 0, False, None), (3, 2, 3, 1, 77, 76, True, (77, 20)), (2, 3, 2, 49, 49, 0, False, (49, 0, 7)), (3, 1, 4, 130, 259, 129, True, None),
         (2, 2, 1, 300, 70, 0, True, (70, 64)), (5, 1, 2, 65, 65, -3, True, (65,)), (8, 1, 2, 33, 513, 7, True, (500,)), (4, 2, 2, 100, 31, 0, False, (31, 30)),
         (2, 2, 2, 8, 40, -9, True, (40, 2)), (2, 1, 1, 600, 600, 0, True, None), (7, 2, 1, 3, 1000, 0, False, (1000, 999)), (6, 1, 1, 257, 255, 100, True, None)]


@BITS
@pytest.mark.parametrize("case", PAIRS, ids=str)
@pytest.mark.parametrize("reach,buckets", [(20, 32), (0, 1), (600, 64)])
def test_bias_and_its_gradient(case, bits, reach, buckets):
    n, batch, heads, Q, K, first, causal, lengths = case
    ring = RINGS[bits][0]
    rng = np.random.default_rng(Q + K + reach)
    lut = rng.integers(0, buckets, size=2 * reach + 1).astype(np.int32)
    if reach:
        lut[1], lut[-2] = -1, buckets
    x, table = uniform(rng, bits, n, batch, heads, Q, K), uniform(rng, bits, n, heads, buckets)
    kw = dict(first=first, causal=causal)
    lens = None if lengths is None else ints(lengths)
    for f in (0, 9):
        tup = tuple_of(rng, bits, x.shape) if f else None
        want = gen.relbias_trunc(x, table, lut, f, tup, lengths=lengths, masked=(1 << bits) - 99, **kw)
        xd, td = dev(x), tup and [dev(t) for t in tup]
        got = ring.relbias_trunc(xd, dev(table), ints(lut), f=f, tuple_=td, lengths=lens, masked=-99, **kw)
        assert same(got, want)
        ring.relbias_trunc(xd, dev(table), ints(lut), f=f, tuple_=td, lengths=lens, masked=-99, out=xd, **kw)
        assert same(xd, want)
    dirty = torch.full((n, heads, buckets), 77, dtype=xd.dtype, device="cuda")
    assert same(ring.relbias_grad(dev(x), ints(lut), buckets, lengths=lens, out=dirty, **kw), gen.relbias_grad(x, lut, buckets, lengths=lengths, **kw))


def test_gradient_is_the_difference_on_the_gpu():
    """The bias is linear: one more in a bucket changes sum(w * out) by the gradient for dS = w, exactly."""
    rng = np.random.default_rng(5)
    n, batch, heads, Q, K, buckets = 2, 2, 3, 70, 90, 16
    lut = ints(spin.relative_buckets(buckets, 40, True))
    x, w, table = dev(uniform(rng, 64, n, batch, heads, Q, K)), dev(uniform(rng, 64, n, batch, heads, Q, K)), dev(uniform(rng, 64, n, heads, buckets))
    lengths = ints([90, 31])
    grad = spin.relbias_grad(w, lut, buckets, lengths=lengths)
    base = spin.relbias_trunc(x, table, lut, lengths=lengths)
    for k in range(buckets):
        more = table.clone()
        more[:, :, k] += 1
        d = spin.relbias_trunc(x, more, lut, lengths=lengths) - base
        assert torch.equal((w * d).sum((1, 3, 4)), grad[:, :, k])


@BITS
def test_on_another_stream(bits):
    calls = [run_scores(attention_case("page_ends_inside", bits), bits)[:2], run_values(attention_case("longer", bits), bits)]
    stream = torch.cuda.Stream()
    for call, want in calls:
        with torch.cuda.stream(stream):
            torch.cuda._sleep(2_000_000)                      # inputs are made on this stream, behind this
            got = call()
        stream.synchronize()
        assert same(got, want)


def test_in_a_graph():
    c = attention_case("page_ends_inside", 64)
    rng = c["rng"]
    n, batch, heads, nodes = c["rows"]
    columns, dim = c["columns"], c["dim"]
    shapes = (c["rows"] + (dim,), c["rows"] + (dim,), c["rows"] + (columns,), c["rows"] + (columns,), c["rows"] + (dim,))
    lut, bias = ints(spin.relative_buckets(32, 20, False)), dev(uniform(rng, 64, n, heads, 32))
    pool, table, context, tree = dev(c["pool"]), ints(c["table"]), ints(c["context"]), dev(c["tree"])
    dS = dev(uniform(rng, 64, n, 2, heads, 40, 40))
    ops = [dev(uniform(rng, 64, *s)) for s in shapes]

    def step():
        Q, A, C, A2, C2 = ops
        S = spin.cache_scores(pool, table, context, Q, A, C, tree=tree, masked=5, bias=(bias, lut))
        return S, spin.cache_values(pool, table, context, S, A2, C2, tree=tree), spin.relbias_grad(dS, lut, 32, causal=True)
    want = [t.clone() for t in step()]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step()
    for k in range(4):
        if k == 2:                                            # other inputs in the same buffers
            for t in ops:
                t += 12345
            dS.neg_()
        want = [t.clone() for t in step()]
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want)), k


def test_offsets_past_32_bits():
    """A pool of 2^32 + 2^22 words; the sequence lives on its last pages."""
    n, tokens, dim, pages = 1, 4096, 256, 2050
    rng = np.random.default_rng(8)
    K = torch.empty((n + 1, pages, 1, tokens, dim), dtype=torch.int32, device="cuda")
    assert K.numel() > 1 << 32
    small = uniform(rng, 32, n + 1, 4, 1, tokens, dim)
    K[:, -4:] = dev(small)
    table, near = np.array([[pages - 2, pages - 1]], np.int32), np.array([[2, 3]], np.int32)
    context, nodes, columns = np.array([4093]), 3, 4096 + 9
    tree = dev(np.array([[1, 3, 7]]))
    Q, A, C = uniform(rng, 32, n, 1, 2, nodes, dim), uniform(rng, 32, n, 1, 2, nodes, dim), uniform(rng, 32, n, 1, 2, nodes, columns)
    got = spin.ring32.cache_scores(K, ints(table), ints(context), dev(Q), dev(A), dev(C), tree=tree)
    assert same(got, gen.scores(small, near, context, Q, A, C, tree=np.array([[1, 3, 7]])))
    P, A2, C2 = uniform(rng, 32, *C.shape), uniform(rng, 32, *C.shape), uniform(rng, 32, *Q.shape)
    got = spin.ring32.cache_values(K, ints(table), ints(context), dev(P), dev(A2), dev(C2), tree=tree)
    assert same(got, gen.values(small, near, context, P, A2, C2, tree=np.array([[1, 3, 7]])))
    x, b = uniform(rng, 32, n, 1, 1, 7, dim), uniform(rng, 32, n, 1, 1, 7, dim)
    small = gen.append(small, near, [4092], None, x, b)
    pools = spin.ring32.cache_append((K, K), ints(table), ints([4092]), (dev(x),) * 2, (dev(b),) * 2)
    small = gen.copy(small, [3], [0])
    spin.ring32.cache_copy(pools, ints([pages - 1]), ints([pages - 4]))
    torch.cuda.synchronize()
    assert same(K[:, -4:], small)


@BITS
@pytest.mark.parametrize("n,dim,context", [(8, 256, 130), (3, 128, 700)])
def test_largest_sums_of_scores(bits, n, dim, context):
    """Every digit of every factor is -128, so the int32 diagonals are as large as they get; the words have a closed form."""
    ring, unsigned, _ = RINGS[bits]
    w = int(-(0x8080808080808080 % (1 << bits))) % (1 << bits)
    word = dev(np.array([w], unsigned))
    heads, nodes, columns = 4, 5, context + 5
    pool = word.expand((n + 1, 1, 1, 1024, dim)).contiguous()
    A = word.expand((n, 1, heads, nodes, dim)).contiguous()
    Q = A.clone()
    Q[0] += word                                              # E = sum (Q - A) = the word
    C = dev(uniform(np.random.default_rng(n), bits, n, 1, heads, nodes, columns))
    got = ring.cache_scores(pool, ints([[0]]), ints([context]), Q, A, C, masked=3)
    seen = torch.arange(columns, device="cuda") <= context + torch.arange(nodes, device="cuda")[:, None]
    want = torch.where(seen, C + 2 * dim * word * word, 0)
    want[0] += torch.where(seen, 0, 3).to(C.dtype)
    assert torch.equal(got, want)
    tup = [dev(uniform(np.random.default_rng(n + k), bits, *C.shape)) for k in range(3)]
    got = ring.cache_scores(pool, ints([[0]]), ints([context]), Q, A, C, f=9, tuple_=tup, masked=3)
    want = torch.where(seen, ring.trunc((C + 2 * dim * word * word).view(n, -1), *[t.view(n, -1) for t in tup], 9).view(C.shape), 0)
    want[0] += torch.where(seen, 0, 3).to(C.dtype)
    assert torch.equal(got, want)


@BITS
@pytest.mark.parametrize("n,nodes,dim", [(8, 1, 128), (3, 3, 128), (1, 1, 64)])
def test_largest_sums_of_values(bits, n, nodes, dim):
    """The same over the longest ranges that a workgroup sums in int32 (all pages of the table are one page)."""
    ring, unsigned, _ = RINGS[bits]
    w = int(-(0x8080808080808080 % (1 << bits))) % (1 << bits)
    word = dev(np.array([w], unsigned))
    batch, heads, context = 4, 8, 32768 - nodes
    pool = word.expand((n + 1, 1, heads, 1024, dim)).contiguous()
    A = word.expand((n, batch, heads, nodes, context + nodes)).contiguous()
    P = A.clone()
    P[0] += word
    C = dev(uniform(np.random.default_rng(n), bits, n, batch, heads, nodes, dim))
    table = torch.zeros((batch, 32), dtype=torch.int32, device="cuda")
    count = (context + 1 + torch.arange(nodes, device="cuda")).to(C.dtype)[:, None]
    plain = C + 2 * count * word * word
    assert torch.equal(ring.cache_values(pool, table, ints([context] * batch), P, A, C), plain)
    tup = [dev(uniform(np.random.default_rng(n + k), bits, *C.shape)) for k in range(3)]
    got = ring.cache_values(pool, table, ints([context] * batch), P, A, C, f=9, tuple_=tup)
    assert torch.equal(got, ring.trunc(plain.view(n, -1), *[t.view(n, -1) for t in tup], 9).view(C.shape))


@pytest.mark.parametrize("n,heads,dim,context", [(2, 1, 128, 150), (3, 2, 112, 17)])
def test_values_of_a_wide_call_with_short_contexts(n, heads, dim, context):
    """Columns for a cache larger than the chip keeps (read with non-temporal loads), most of them past the table."""
    rng = np.random.default_rng(dim)
    columns, nodes = (1 << 28) // (8 * (n + 1) * heads * dim) + 77, 2
    pool, table = uniform(rng, 64, n + 1, 14, heads, 16, dim), table_of(rng, 1, 12, 14)
    P, A = uniform(rng, 64, n, 1, heads, nodes, columns), uniform(rng, 64, n, 1, heads, nodes, columns)
    C, tree = uniform(rng, 64, n, 1, heads, nodes, dim), np.array([[1, 3]])
    tup = tuple_of(rng, 64, C.shape)
    short = 12 * 16 + 3                                       # nothing beyond the table is seen
    want = gen.values(pool, table, np.array([context]), P[..., :short], A[..., :short], C, 16, tup, tree)
    got = spin.cache_values(dev(pool), ints(table), ints([context]), dev(P), dev(A), dev(C), f=16, tuple_=[dev(t) for t in tup], tree=dev(tree))
    assert same(got, want)


@BITS
@pytest.mark.parametrize("n,heads,nodes,dim", [(2, 1, 1, 128), (3, 1, 2, 72), (2, 4, 3, 128), (5, 3, 5, 40)])
def test_scores_of_a_wide_call_with_short_contexts(bits, n, heads, nodes, dim):
    """The same for keys, by words (up to two rows) and by digits."""
    ring, unsigned, _ = RINGS[bits]
    rng = np.random.default_rng(dim + nodes)
    columns, context = (1 << 31) // (bits * (n + 1) * dim) + 77, 150
    pool, table = uniform(rng, bits, n + 1, 14, 1, 16, dim), table_of(rng, 1, 12, 14)
    Q, A = uniform(rng, bits, n, 1, heads, nodes, dim), uniform(rng, bits, n, 1, heads, nodes, dim)
    C = uniform(rng, bits, n, 1, heads, nodes, columns)
    tup = tuple_of(rng, bits, C.shape)
    short = 12 * 16 + 3
    want = gen.scores(pool, table, np.array([context]), Q, A, C[..., :short], 9, tuple(t[..., :short] for t in tup), masked=5)
    got = ring.cache_scores(dev(pool), ints(table), ints([context]), dev(Q), dev(A), dev(C), f=9, tuple_=[dev(t) for t in tup], masked=5)
    assert same(got[..., :short].contiguous(), want)
    assert (got[0, ..., short:] == 5).all() and not got[1:, ..., short:].any()


@BITS
@pytest.mark.parametrize("n,heads,nodes,dim", [(2, 2, 2, 128), (2, 1, 5, 128), (3, 4, 4, 112), (2, 3, 7, 256)])
def test_values_of_a_wide_call_by_rows(bits, n, heads, nodes, dim):
    """Values for a cache larger than the chip keeps, of four, five, 16 and 21 rows a cached head."""
    ring, unsigned, _ = RINGS[bits]
    rng = np.random.default_rng(dim + nodes)
    columns, context = (1 << 31) // (bits * (n + 1) * dim) + 77, 171
    pool, table = uniform(rng, bits, n + 1, 14, 1, 16, dim), table_of(rng, 1, 12, 14)
    P, A = uniform(rng, bits, n, 1, heads, nodes, columns), uniform(rng, bits, n, 1, heads, nodes, columns)
    C = uniform(rng, bits, n, 1, heads, nodes, dim)
    tup, short = tuple_of(rng, bits, C.shape), 12 * 16 + 3
    want = gen.values(pool, table, np.array([context]), P[..., :short], A[..., :short], C, 9, tup)
    got = ring.cache_values(dev(pool), ints(table), ints([context]), dev(P), dev(A), dev(C), f=9, tuple_=[dev(t) for t in tup])
    assert same(got, want)


@BITS
@pytest.mark.parametrize("f", [0, 9])
@pytest.mark.parametrize("n,share,nodes", [(1, 1, 1), (3, 2, 1), (8, 1, 2), (2, 1, 4), (5, 3, 1), (4, 4, 1)])
@pytest.mark.parametrize("dim", [8, 24, 40, 72, 104, 136, 200, 256])
def test_few_rows(bits, f, n, share, nodes, dim):
    """One to four rows a cached head, heads of every kind of length, a page that is not there, sequences of none to some hundred tokens."""
    ring, unsigned, _ = RINGS[bits]
    rng = np.random.default_rng(dim * 31 + n)
    heads, contexts = 2 * share, [0, 3, 150, 333, -1]
    pool, table = uniform(rng, bits, n + 1, 120, 2, 16, dim), table_of(rng, len(contexts), 22, 120)
    table[2, 4], table[3, 0] = -1, 120
    columns = max(contexts) + nodes + 2
    Q, A = (uniform(rng, bits, n, len(contexts), heads, nodes, dim) for _ in range(2))
    C = uniform(rng, bits, n, len(contexts), heads, nodes, columns)
    tup = tuple_of(rng, bits, C.shape) if f else None
    tree = rng.integers(0, 1 << nodes, (len(contexts), nodes))
    ctx = np.array(contexts)
    put = (lambda t: None if t is None else [dev(x) for x in t])
    want = gen.scores(pool, table, ctx, Q, A, C, f, tup, tree, masked=7)
    assert same(ring.cache_scores(dev(pool), ints(table), ints(contexts), dev(Q), dev(A), dev(C), f=f, tuple_=put(tup), tree=dev(tree), masked=7), want)
    P, A = (uniform(rng, bits, n, len(contexts), heads, nodes, columns) for _ in range(2))
    C = uniform(rng, bits, n, len(contexts), heads, nodes, dim)
    tup = tuple_of(rng, bits, C.shape) if f else None
    want = gen.values(pool, table, ctx, P, A, C, f, tup, tree)
    assert same(ring.cache_values(dev(pool), ints(table), ints(contexts), dev(P), dev(A), dev(C), f=f, tuple_=put(tup), tree=dev(tree)), want)
