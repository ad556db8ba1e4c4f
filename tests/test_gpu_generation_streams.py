"""Every cache, attention and bias call on a stream of its own and in a graph, through the compiled binding and through ctypes."""
import pytest
import torch

from paper_2402_02320_amd import spin
from test_gpu_generation import RINGS, ints

pytestmark = pytest.mark.gpu
BITS = pytest.mark.parametrize("bits", [64, 32])
N, BATCH, KV, HEADS, NODES, DIM, TOKENS, COLUMNS = 3, 2, 2, 6, 3, 72, 16, 150


class Step:
    """One of each call on operands that stay where they are: name -> (an operand that is written late, call, tensors of the result)."""

    def __init__(self, bits, seed):
        self.ring, self.bits = RINGS[bits][0], bits
        torch.manual_seed(seed)
        lead = (N, BATCH, HEADS, NODES)
        self.table = ints([[4, 9, 1, 0, 7, 11, 3, 5, 2, 8], [10, 12, 6, 13, 19, 14, 18, 15, 17, 16]])
        self.context, self.count = ints([147, 90]), ints([5, 2])
        self.src, self.dst = ints([20, 21]), ints([22, 23])
        self.kept, self.kept_count = ints([[1, 2, 0], [2, 0, 0]]), ints([2, 1])
        self.tree = torch.tensor([[1, 3, 5], [1, 2, 6]], device="cuda")
        self.depth, self.lut, self.bias = ints([[0, 1, 1], [0, 0, 2]]), spin.relative_buckets(32, 20, False).cuda(), self.u(N, HEADS, 32)
        self.K, self.V = self.u(N + 1, 24, KV, TOKENS, DIM), self.u(N + 1, 24, KV, TOKENS, DIM)
        self.x, self.b = [[self.u(N, BATCH, KV, 5, DIM) for _ in range(2)] for _ in range(2)]
        self.Q, self.A, self.C, self.tup = self.u(*lead, DIM), self.u(*lead, DIM), self.u(*lead, COLUMNS), [self.u(*lead, COLUMNS) for _ in range(3)]
        self.P, self.AP, self.CP, self.tupP = self.u(*lead, COLUMNS), self.u(*lead, COLUMNS), self.u(*lead, DIM), [self.u(*lead, DIM) for _ in range(3)]
        self.S, self.tupS, self.lengths = self.u(N, BATCH, HEADS, 40, 130), [self.u(N, BATCH, HEADS, 40, 130) for _ in range(3)], ints([130, 61])
        self.pools = {k: (self.K.clone(), self.V.clone()) for k in ("append", "copy", "compact")}

    def u(self, *s):
        return torch.empty(s, dtype=torch.int64 if self.bits == 64 else torch.int32, device="cuda").random_(-2 ** (self.bits - 1), 2 ** (self.bits - 1) - 1)

    def calls(self):
        r, kw = self.ring, dict(first=90, causal=True, lengths=self.lengths)
        return {
            "append": (self.x[0], lambda: r.cache_append(self.pools["append"], self.table, self.context, self.x, self.b, count=self.count)),
            "copy": (self.pools["copy"][0], lambda: r.cache_copy(self.pools["copy"], self.src, self.dst)),
            "compact": (self.pools["compact"][1], lambda: r.cache_compact(self.pools["compact"], self.table, self.context, self.kept, self.kept_count)),
            "scores": (self.Q, lambda: r.cache_scores(self.K, self.table, self.context, self.Q, self.A, self.C, f=9, tuple_=self.tup, tree=self.tree, masked=5,
                                                      bias=(self.bias, self.lut), depth=self.depth)),
            "values": (self.P, lambda: r.cache_values(self.V, self.table, self.context, self.P, self.AP, self.CP, f=9, tuple_=self.tupP, tree=self.tree)),
            "bias": (self.S, lambda: r.relbias_trunc(self.S, self.bias, self.lut, f=9, tuple_=self.tupS, masked=7, **kw)),
            "grad": (self.S, lambda: r.relbias_grad(self.S, self.lut, 32, **kw)),
        }


def tensors(result):
    return [t.clone() for t in (result if isinstance(result, (list, tuple)) else [result])]


@BITS
@pytest.mark.parametrize("fast", [True, False], ids=["binding", "ctypes"])
@pytest.mark.parametrize("name", ["append", "copy", "compact", "scores", "values", "bias", "grad"])
def test_behind_work_of_another_stream(bits, fast, name, monkeypatch):
    """An operand gets its words on the side stream, late, and nothing between that and the call makes the host wait: a call on any other stream would
    read the words that were there before."""
    if not fast:
        spin.lib()
        monkeypatch.setattr(spin, "_fast", None)
    operand, call = Step(bits, 1).calls()[name]
    late = torch.randint_like(operand, -2 ** 31, 2 ** 31 - 1)
    operand.copy_(late)
    want = tensors(call())
    operand, call = Step(bits, 1).calls()[name]
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):                           # the call's own memory and kernels are there
        Step(bits, 2).calls()[name][1]()
    torch.cuda.synchronize()
    with torch.cuda.stream(stream):
        torch.cuda._sleep(20_000_000)
        operand.copy_(late)
        got = call()
    pending = not stream.query()                              # the host was not made to wait
    stream.synchronize()
    assert pending
    got = tensors(got)
    assert len(got) == len(want) and all(torch.equal(a, b) for a, b in zip(got, want))


@BITS
def test_all_calls_in_a_graph(bits):
    """Several replays with eager work of the same program between them, each against the eager calls on the same words."""
    s = Step(bits, 3)
    calls = s.calls()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for _, call in calls.values():
            call()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = {k: call() for k, (_, call) in calls.items()}
    for turn in range(5):
        if turn > 1:
            for t in (s.Q, s.P, s.S, s.x[0], s.b[1], s.K, s.V):
                t += 12345 + turn
        before = {k: [p.clone() for p in v] for k, v in s.pools.items()}
        want = {k: tensors(call()) for k, (_, call) in calls.items()}
        torch.cuda.synchronize()
        for k, v in s.pools.items():
            for p, q in zip(v, before[k]):
                p.copy_(q)
        graph.replay()
        torch.cuda.synchronize()
        for k in calls:
            assert all(torch.equal(a, b) for a, b in zip(tensors(got[k]), want[k])), (turn, k)
