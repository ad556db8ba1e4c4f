"""The cache, attention and bias calls through the compiled binding and through ctypes: the same words, the same `out` object; and what only the long way takes."""
import pytest
import torch

from paper_2402_02320_amd import spin

pytestmark = pytest.mark.gpu


def u(bits, *s):
    dtype = torch.int64 if bits == 64 else torch.int32
    return torch.empty(s, dtype=dtype, device="cuda").random_(-2 ** (bits - 1), 2 ** (bits - 1) - 1)


def i32(*v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def calls(bits):
    ring = spin if bits == 64 else spin.ring32
    torch.manual_seed(7)
    pools = [u(bits, 3, 9, 2, 16, 40) for _ in range(2)]
    table, context = i32([8, 1, 2, 3], [4, 0, 6, 7]), i32(50, 33)
    rows = [u(bits, 2, 2, 2, 5, 40) for _ in range(4)]
    narrow, wide = [u(bits, 2, 2, 6, 3, 40) for _ in range(6)], [u(bits, 2, 2, 6, 3, 53) for _ in range(6)]
    tree = torch.tensor([[1, 3, 5], [1, 2, 4]], device="cuda")
    lut, bias, depth = i32(*range(21)), u(bits, 2, 6, 21), i32([0, 1, 1], [0, 0, 0])
    x = [u(bits, 2, 2, 6, 30, 41) for _ in range(4)]
    copied = [p.clone() for p in pools]
    return {
        "append": lambda: ring.cache_append(tuple(p.clone() for p in pools), table, context, rows[:2], rows[2:], count=i32(5, 2)),
        "append_all": lambda: ring.cache_append([p.clone() for p in pools], table, context, tuple(rows[:2]), tuple(rows[2:])),
        "copy": lambda: ring.cache_copy([p.clone() for p in pools], i32(1, 2), i32(5, 8)),
        "compact": lambda: ring.cache_compact([p.clone() for p in copied], table, context, i32([1, 2, 0], [0, 2, 0]), i32(2, 2)),
        "scores": lambda: ring.cache_scores(pools[0], table, context, *narrow[:2], wide[0], f=9, tuple_=wide[1:4], tree=tree, masked=-5, bias=(bias, lut), depth=depth),
        "scores_plain": lambda: ring.cache_scores(pools[0], table, context, *narrow[:2], wide[0], masked=1 << 70),
        "values": lambda: ring.cache_values(pools[1], table, context, *wide[:2], narrow[0], f=9, tuple_=tuple(narrow[1:4]), tree=tree),
        "values_plain": lambda: ring.cache_values(pools[1], table, context, *wide[:2], narrow[0], workspace=torch.empty(1 << 20, dtype=torch.uint8, device="cuda")),
        "bias": lambda: ring.relbias_trunc(x[0], bias, lut, f=9, tuple_=x[1:], first=3, causal=True, lengths=i32(41, 7), masked=-5),
        "bias_plain": lambda: ring.relbias_trunc(x[0], bias, lut),
        "grad": lambda: ring.relbias_grad(x[0], lut, 21, first=-1, causal=True, lengths=i32(41, 7)),
    }


NAMES = ["append", "append_all", "copy", "compact", "scores", "scores_plain", "values", "values_plain", "bias", "bias_plain", "grad"]


@pytest.mark.parametrize("bits", [64, 32])
@pytest.mark.parametrize("name", NAMES)
def test_same_words_both_ways(name, bits, monkeypatch):
    spin.lib()
    call, taken, fast = calls(bits)[name], [], spin._fast

    class Watch:
        def __getattr__(self, entry):
            def made(*a):
                taken.append(getattr(fast, entry)(*a))
                return taken[-1]
            return made
    monkeypatch.setattr(spin, "_fast", Watch())
    got = call()
    assert len(taken) == 1 and taken[0] is got                # the compiled binding took it
    monkeypatch.setattr(spin, "_fast", None)
    want = call()
    got, want = (list(v) if isinstance(v, (list, tuple)) else [v] for v in (got, want))
    assert len(got) == len(want) and all(torch.equal(a, b) and a.dtype == b.dtype for a, b in zip(got, want))


def test_out_is_returned_and_refusals_are_the_same():
    ring = spin
    c = calls(64)
    want = c["scores_plain"]()
    o = torch.empty_like(want)
    torch.manual_seed(7)
    pool, table, context = u(64, 3, 9, 2, 16, 40), i32([8, 1, 2, 3], [4, 0, 6, 7]), i32(50, 33)
    Q, C = u(64, 2, 2, 6, 3, 40), u(64, 2, 2, 6, 3, 53)
    assert ring.cache_scores(pool, table, context, Q, Q, C, out=o) is o
    x, lut, bias = u(64, 2, 2, 6, 30, 41), i32(*range(21)), u(64, 2, 6, 21)
    assert ring.relbias_trunc(x, bias, lut, out=x) is x
    for bad in (lambda: ring.cache_scores(pool, table, context, Q, Q, C, f=62, tuple_=[C] * 3), lambda: ring.cache_scores(pool, table, context.long(), Q, Q, C),
                lambda: ring.cache_scores(pool, table, context[:1], Q, Q, C), lambda: ring.cache_scores(pool, table, context, Q, Q, C[..., :50]),
                lambda: ring.cache_scores(pool.transpose(2, 3), table, context, Q, Q, C), lambda: ring.cache_scores(pool.int(), table, context, Q, Q, C),
                lambda: ring.cache_values(pool, table, context, C, C, Q, workspace=torch.empty(16, dtype=torch.uint8, device="cuda")[:0]),
                lambda: ring.cache_scores(pool, table, context, Q, Q, C, out=o[:1]), lambda: ring.relbias_grad(x, lut[:20], 21), lambda: ring.relbias_grad(x, lut, 1025),
                lambda: ring.cache_copy((pool, pool[:, :5].contiguous()), i32(1), i32(2)), lambda: ring.cache_copy((pool, pool.cpu()), i32(1), i32(2))):
        with pytest.raises(spin.SpinError):
            bad()
