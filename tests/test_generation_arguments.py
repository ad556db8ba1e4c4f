"""What the cache, attention and bias calls refuse, on the CPU: the C entry points before any launch, and the Python binding before the library."""
import ctypes

import pytest
import torch

from paper_2402_02320_amd import spin
from test_binding_arguments import Record, WS

EINVAL, ERANGE, EWORKSPACE = 1, 2, 3
P, ODD = 0x10000, 0x10004


@pytest.fixture(scope="module")
def L():
    return spin.lib()


def cache(**kw):
    d = dict(n=2, pages=8, heads=4, page_tokens=16, dim=64, K=P, V=P, batch=2, table_pages=3, table=P)
    d.update(kw)
    return ctypes.byref(spin._Cache(*[d[k] for k, _ in spin._Cache._fields_]))


def bias(**kw):
    d = dict(buckets=32, reach=128, bucket_of=P, table=P)
    d.update(kw)
    return ctypes.byref(spin._RelBias(*[d[k] for k, _ in spin._RelBias._fields_]))


BAD_CACHES = [(dict(n=0), EINVAL), (dict(n=9), EINVAL), (dict(pages=0), EINVAL), (dict(heads=0), EINVAL), (dict(dim=0), EINVAL), (dict(dim=12), EINVAL),
              (dict(dim=264), EINVAL), (dict(page_tokens=8), EINVAL), (dict(page_tokens=48), EINVAL), (dict(page_tokens=8192), EINVAL),
              (dict(page_tokens=-16), EINVAL), (dict(pages=1 << 30, heads=64), ERANGE)]
BAD_TABLES = [(dict(batch=0), EINVAL), (dict(table_pages=0), EINVAL), (dict(table=None), EINVAL), (dict(table=P + 2), EINVAL), (dict(batch=20000), ERANGE)]


@pytest.mark.parametrize("pre", ["spin_", "spin32_"])
def test_refusals_of_the_upkeep(L, pre):
    app, cop, com = (getattr(L, pre + "cache_" + k) for k in ("append", "copy", "compact"))

    def append(c, rows=1, start=P, count=P, x=(P,) * 4):
        return app(c, rows, start, count, *x, None)
    for kw, st in BAD_CACHES + BAD_TABLES:
        assert append(cache(**kw)) == st and com(cache(**kw), 4, P, P, P, None) == st, kw
    for kw, st in BAD_CACHES:
        assert cop(cache(**kw), 4, P, P, None) == st, kw
    for k in ("K", "V"):
        for v in (None, ODD):
            assert append(cache(**{k: v})) == cop(cache(**{k: v}), 4, P, P, None) == com(cache(**{k: v}), 4, P, P, P, None) == EINVAL
    assert append(None) == cop(None, 4, P, P, None) == com(None, 4, P, P, P, None) == EINVAL
    assert append(cache(), rows=0) == append(cache(), start=None) == append(cache(), start=P + 1) == append(cache(), count=P + 2) == EINVAL
    assert append(cache(), rows=(1 << 24) + 1) == ERANGE
    for i in range(4):
        for bad in (None, ODD):
            assert append(cache(), x=(P,) * i + (bad,) + (P,) * (3 - i)) == EINVAL
    assert cop(cache(), 0, P, P, None) == cop(cache(), 4, None, P, None) == cop(cache(), 4, P, None, None) == EINVAL
    assert cop(cache(), 65536, P, P, None) == ERANGE
    for nodes in (0, 65):
        assert com(cache(), nodes, P, P, P, None) == EINVAL
    for lists in ((None, P, P), (P, None, P), (P, P, None)):
        assert com(cache(), 4, *lists, None) == EINVAL


@pytest.mark.parametrize("pre,most", [("spin_", 61), ("spin32_", 29)])
def test_refusals_of_the_attention(L, pre, most):
    sc, va, need = (getattr(L, pre + "cache_" + k) for k in ("scores", "values", "values_workspace_bytes"))

    def both(c=None, heads=8, nodes=4, columns=40, f=9, context=P, tree=P, ops=(P,) * 7, bad=EINVAL, values_too=True, ws=P, size=1 << 40):
        q, a, cc, r, rt, rm, out = ops
        assert sc(c or cache(V=None), heads, nodes, columns, f, context, tree, q, a, cc, r, rt, rm, 5, bias(), P, out, None) == bad
        if values_too:
            assert va(c or cache(K=None), heads, nodes, columns, f, context, tree, q, a, cc, r, rt, rm, out, ws, size, None) == bad
    for kw, st in BAD_CACHES + BAD_TABLES:
        both(cache(**kw), bad=st)
        assert need(cache(**kw), 8, 4, 40) == 0
    for kw in (dict(heads=0), dict(heads=6), dict(nodes=0), dict(nodes=65), dict(columns=0), dict(f=-1), dict(f=most + 1), dict(context=None),
               dict(context=P + 2), dict(tree=ODD)):
        both(**kw)
    both(columns=(1 << 24) + 1, bad=ERANGE)
    both(heads=1 << 16, nodes=1, bad=ERANGE)
    for i in range(7):
        for bad in (None, ODD):
            both(ops=(P,) * i + (bad,) + (P,) * (6 - i))
    assert need(cache(), 6, 4, 40) == need(cache(), 8, 65, 40) == need(cache(), 8, 4, 0) == need(None, 8, 4, 40) == 0
    size = need(cache(), 8, 4, 40)
    assert size > 0

    def values(ws, size):
        return va(cache(), 8, 4, 40, 0, P, None, P, P, P, None, None, None, P, ws, size, None)
    assert values(None, size) == values(P + 128, size) == values(P, size - 1) == EWORKSPACE
    for kw in (dict(buckets=0), dict(buckets=1025), dict(reach=-1), dict(reach=1 << 16), dict(bucket_of=None), dict(bucket_of=P + 1), dict(table=None), dict(table=ODD)):
        assert sc(cache(), 8, 4, 40, 0, P, None, P, P, P, None, None, None, 5, bias(**kw), P, P, None) == EINVAL, kw
    assert sc(cache(), 8, 4, 40, 0, P, None, P, P, P, None, None, None, 5, bias(), P + 2, P, None) == EINVAL


@pytest.mark.parametrize("pre,most", [("spin_", 61), ("spin32_", 29)])
def test_refusals_of_the_bias(L, pre, most):
    tr, gr = getattr(L, pre + "relbias_trunc"), getattr(L, pre + "relbias_grad")

    def both(dims=(2, 2, 4, 8, 8), first=0, lengths=None, bad=EINVAL):
        assert tr(*dims, first, 1, lengths, 9, P, P, P, P, 5, bias(), P, None) == gr(*dims, first, 1, lengths, P, bias(), P, None) == bad, dims
    for i in range(5):
        both((2, 2, 4, 8, 8)[:i] + (0,) + (2, 2, 4, 8, 8)[i + 1:])
    both((9, 2, 4, 8, 8))
    both(lengths=P + 2)
    for dims in ((2, 1 << 14, 4, 8, 8), (2, 2, 4, (1 << 24) + 1, 8), (2, 2, 4, 8, (1 << 24) + 1), (8, 60, 1000, 1 << 20, 1 << 20)):
        both(dims, bad=ERANGE)
    both(first=1 << 29, bad=ERANGE)
    both(first=-(1 << 29), bad=ERANGE)
    d = (2, 2, 4, 8, 8, 0, 0, None)
    for f in (-1, most + 1):
        assert tr(*d, f, P, P, P, P, 5, bias(), P, None) == EINVAL
    for i in range(5):
        x = [P] * 5
        x[i] = None
        assert tr(*d, 9, *x[:4], 5, bias(), x[4], None) == EINVAL
    for kw in (dict(buckets=0), dict(reach=-1), dict(bucket_of=None), dict(table=None)):
        assert tr(*d, 9, P, P, P, P, 5, bias(**kw), P, None) == EINVAL
        if "table" not in kw:
            assert gr(*d, P, bias(**kw), P, None) == EINVAL
    assert tr(*d, 9, P, P, P, P, 5, None, P, None) == gr(*d, P, None, P, None) == gr(*d, None, bias(), P, None) == gr(*d, P, bias(), ODD, None) == EINVAL


# ---- the binding ---------------------------------------------------------------------------------------------------
@pytest.fixture
def record(monkeypatch):
    r = Record()
    monkeypatch.setattr(spin, "_lib", r)
    monkeypatch.setattr(spin, "_fast", None)
    monkeypatch.setattr(spin, "_dev", lambda t, name: t.data_ptr())
    monkeypatch.setattr(spin, "_dev32", lambda t, name: t.data_ptr())
    monkeypatch.setattr(spin, "_stream", lambda: 0)
    real = spin._list32

    class OnGpu(torch.Tensor):
        is_cuda = True
    monkeypatch.setattr(spin, "_list32", lambda t, name, *shape: real(t.as_subclass(OnGpu), name, *shape))
    monkeypatch.setattr(spin._Word, "_tree", staticmethod(lambda t, b, m: None if t is None else spin._shapes(tuple(t.shape) == (b, m))))
    return r


def w(*shape):
    return torch.zeros(shape, dtype=torch.int64)


def i32(*shape):
    return torch.zeros(shape, dtype=torch.int32)


POOL, ROWS = (3, 5, 2, 16, 8), (2, 4, 2, 6, 8)                # two parties, four sequences, two cached heads
GOOD = {
    "cache_append": (((w(*POOL), w(*POOL)), i32(4, 3), i32(4), (w(*ROWS), w(*ROWS)), (w(*ROWS), w(*ROWS))), {}),
    "cache_copy": (((w(*POOL), w(*POOL)), i32(3), i32(3)), {}),
    "cache_compact": (((w(*POOL), w(*POOL)), i32(4, 3), i32(4), i32(4, 7), i32(4)), {}),
    "cache_scores": ((w(*POOL), i32(4, 3), i32(4), w(2, 4, 6, 3, 8), w(2, 4, 6, 3, 8), w(2, 4, 6, 3, 20)),
                     dict(f=9, tuple_=[w(2, 4, 6, 3, 20)] * 3, tree=w(4, 3), bias=(w(2, 6, 32), i32(21)), depth=i32(4, 3))),
    "cache_values": ((w(*POOL), i32(4, 3), i32(4), w(2, 4, 6, 3, 20), w(2, 4, 6, 3, 20), w(2, 4, 6, 3, 8)),
                     dict(f=9, tuple_=[w(2, 4, 6, 3, 8)] * 3, tree=w(4, 3), workspace=WS)),
    "relbias_trunc": ((w(2, 3, 6, 4, 5), w(2, 6, 32), i32(21)), dict(f=9, tuple_=[w(2, 3, 6, 4, 5)] * 3, lengths=i32(3))),
    "relbias_grad": ((w(2, 3, 6, 4, 5), i32(21), 32), dict(lengths=i32(3))),
}


def swapped(name, at, value):
    args, kw = GOOD[name]
    if isinstance(at, str):
        return args, {**kw, at: value}
    return args[:at] + (value,) + args[at + 1:], kw


@pytest.mark.parametrize("name", sorted(GOOD))
def test_well_formed_calls_reach_the_library(record, name):
    args, kw = GOOD[name]
    getattr(spin, name)(*args, **kw)
    getattr(spin.ring32, name)(*args, **kw)
    assert record.launched == ["spin_" + name, "spin32_" + name]


@pytest.mark.parametrize("name,at,value", [
    ("cache_append", 0, (w(*POOL), w(3, 5, 2, 16, 16))), ("cache_append", 0, (w(4, 5, 2, 16, 8),) * 2), ("cache_append", 0, (w(3, 5, 3, 16, 8),) * 2),
    ("cache_append", 1, i32(3, 3)), ("cache_append", 1, w(4, 3)), ("cache_append", 2, i32(3)), ("cache_append", 2, i32(4, 1)), ("cache_append", 3, (w(*ROWS), w(2, 4, 2, 5, 8))),
    ("cache_append", 4, (w(2, 4, 2, 6, 16), w(*ROWS))), ("cache_append", "count", i32(5)),
    ("cache_copy", 1, i32(2)), ("cache_copy", 2, i32(4)), ("cache_copy", 0, (w(*POOL), w(3, 6, 2, 16, 8))),
    ("cache_compact", 1, i32(5, 3)), ("cache_compact", 2, i32(3)), ("cache_compact", 3, i32(4)), ("cache_compact", 3, i32(3, 7)), ("cache_compact", 4, i32(5)),
    ("cache_scores", 0, w(4, 5, 2, 16, 8)), ("cache_scores", 0, w(3, 5, 2, 16, 16)), ("cache_scores", 1, i32(4)), ("cache_scores", 2, i32(3)),
    ("cache_scores", 3, w(2, 4, 6, 2, 8)), ("cache_scores", 4, w(2, 4, 6, 3, 16)), ("cache_scores", 5, w(2, 4, 6, 2, 20)), ("cache_scores", 5, w(2, 4, 6, 3)),
    ("cache_scores", "tuple_", None), ("cache_scores", "tuple_", [w(2, 4, 6, 3, 21)] * 3), ("cache_scores", "tree", w(4, 2)), ("cache_scores", "tree", w(3, 3)),
    ("cache_scores", "bias", (w(2, 5, 32), i32(21))), ("cache_scores", "bias", (w(2, 6, 32), i32(20))), ("cache_scores", "depth", i32(4, 2)),
    ("cache_scores", "out", w(2, 4, 6, 3, 19)),
    ("cache_values", 0, w(4, 5, 2, 16, 8)), ("cache_values", 0, w(3, 5, 2, 16, 16)), ("cache_values", 3, w(2, 4, 6, 3, 21)), ("cache_values", 5, w(2, 4, 6, 2, 8)),
    ("cache_values", "tuple_", None), ("cache_values", "tuple_", [w(2, 4, 6, 3, 20)] * 3), ("cache_values", "tree", w(4, 4)), ("cache_values", "out", w(2, 4, 6, 3, 7)),
    ("relbias_trunc", 0, w(2, 3, 6, 4)), ("relbias_trunc", 1, w(2, 5, 32)), ("relbias_trunc", 1, w(3, 6, 32)), ("relbias_trunc", 2, i32(22)),
    ("relbias_trunc", "tuple_", None), ("relbias_trunc", "tuple_", [w(2, 3, 6, 4, 6)] * 3), ("relbias_trunc", "lengths", i32(4)), ("relbias_trunc", "out", w(2, 3, 6, 4, 4)),
    ("relbias_grad", 0, w(2, 3, 6, 4)), ("relbias_grad", 1, i32(22)), ("relbias_grad", "lengths", i32(2)), ("relbias_grad", "out", w(2, 6, 31)),
])
def test_malformed_calls_are_refused(record, name, at, value):
    args, kw = swapped(name, at, value)
    for ring in (spin, spin.ring32):
        with pytest.raises(spin.SpinError):
            getattr(ring, name)(*args, **kw)
    assert not record.launched


def test_lists_and_words_have_their_types():
    for bad in (torch.zeros(4, dtype=torch.int32), torch.zeros(4, dtype=torch.int64), [1, 2]):
        with pytest.raises(spin.SpinError):
            spin._list32(bad, "context", 4)
    with pytest.raises(spin.SpinError):
        spin.cache_copy((w(*POOL), w(*POOL)), i32(3), i32(3))
    with pytest.raises(spin.SpinError):
        spin._Word._tree(w(4, 3), 4, 3)                       # not on the GPU
