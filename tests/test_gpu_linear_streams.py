"""Every call of linear attention and layer norm on a stream of its own and in a graph, through the compiled binding and through ctypes."""
import pytest
import torch

from paper_2402_02320_amd import spin
from test_gpu_generation import RINGS, ints
from test_gpu_generation_streams import tensors

pytestmark = pytest.mark.gpu
BITS = pytest.mark.parametrize("bits", [64, 32])
N, BATCH, HEADS, TOKENS, KEYS, VALUES, CHUNK, ROWS, DIM = 3, 2, 4, 130, 40, 72, 64, 37, 333
CALLS = ["scores", "states", "outputs", "step", "norm", "norm_grad"]


class Operands:
    """One of each call on operands that stay where they are: name -> (an operand that is written late, call)."""

    def __init__(self, bits, seed):
        self.ring, self.bits = RINGS[bits][0], bits
        torch.manual_seed(seed)
        chunks, lead = -(-TOKENS // CHUNK), (N, BATCH, HEADS)

        def dealt(*s):
            return self.u(*s), [self.u(*s) for _ in range(3)]
        self.kw = dict(f=9, g=6, decay=self.u(HEADS, CHUNK + 1), lengths=ints([TOKENS, 65]))
        self.q, self.k, self.v = [[self.u(*lead, TOKENS, d) for _ in range(2)] for d in (KEYS, KEYS, VALUES)]
        self.P, self.S = [[self.u(*lead, chunks, *s) for _ in range(2)] for s in ((CHUNK, CHUNK), (KEYS, VALUES))]
        self.scores, self.states, self.outputs = dealt(*lead, chunks, CHUNK, CHUNK), dealt(*lead, chunks, KEYS, VALUES), dealt(*lead, TOKENS, VALUES)
        self.state, self.mask = self.u(*lead, KEYS, VALUES), self.u(*lead, KEYS, VALUES)
        self.token = [[self.u(*lead, d) for _ in range(2)] for d in (KEYS, KEYS, VALUES)]
        self.after, self.read = dealt(*lead, KEYS, VALUES), dealt(*lead, VALUES)
        self.once, self.active = self.u(HEADS, 2), ints([1, 0])
        self.x, self.dy, self.xhat = self.u(N, ROWS, DIM), self.u(N, ROWS, DIM), self.u(N, ROWS, DIM)
        self.gamma, self.beta, self.rstd = [self.u(N, DIM) for _ in range(2)], self.u(N, DIM), self.u(N, ROWS)
        self.masks = [self.u(N, ROWS, DIM) for _ in range(3)]
        self.norm = [dealt(N, ROWS, DIM) for _ in range(2)]
        self.row_words, self.grad_words, self.column_words = self.u(N, 60, ROWS), self.u(N, 22, ROWS), self.u(N, 4, DIM)

    def u(self, *s):
        return torch.empty(s, dtype=torch.int64 if self.bits == 64 else torch.int32, device="cuda").random_(-2 ** (self.bits - 1), 2 ** (self.bits - 1) - 1)

    def calls(self):
        r, C, t = self.ring, [c for c, _ in self.norm], [t for _, t in self.norm]
        return {
            "scores": (self.q[0], lambda: r.linattn_scores(self.q, self.k, *self.scores, **self.kw)),
            "states": (self.v[1], lambda: r.linattn_states(self.k, self.v, *self.states, chunk=CHUNK, first=self.state, **self.kw)),
            "outputs": (self.S[0], lambda: r.linattn_outputs(self.P, self.v, self.q, self.S, *self.outputs, **self.kw)),
            "step": (self.state, lambda: r.linattn_step(self.state, *self.token, self.mask, (self.after[0], self.read[0]), (self.after[1], self.read[1]), 9, self.once, 6,
                                                        self.active)),
            "norm": (self.x, lambda: r.layernorm(self.x, self.gamma, self.beta, self.masks[:2], C, t, self.row_words, 9, 15, (768, 128), 1)),
            "norm_grad": (self.rstd, lambda: r.layernorm_grad(self.dy, self.xhat, self.rstd, self.gamma, self.masks, C, t, self.grad_words, self.column_words, 9, 15)),
        }


@BITS
@pytest.mark.parametrize("fast", [True, False], ids=["binding", "ctypes"])
@pytest.mark.parametrize("name", CALLS)
def test_behind_work_of_another_stream(bits, fast, name, monkeypatch):
    """An operand gets its words on the side stream, late, and nothing between that and the call makes the host wait: a call on any other stream would
    read the words that were there before."""
    operand, call = Operands(bits, 1).calls()[name]
    late = torch.randint_like(operand, -2 ** 31, 2 ** 31 - 1)
    operand.copy_(late)
    want = tensors(call())
    if not fast:
        spin.lib()
        monkeypatch.setattr(spin, "_fast", None)
    operand, call = Operands(bits, 1).calls()[name]
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):                           # the call's own memory and kernels are there
        Operands(bits, 2).calls()[name][1]()
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
def test_all_calls_in_two_graphs(bits):
    """Several replays of two graphs, each with memory of its own, with eager work of the same program between them, against the eager calls on the same words."""
    s = Operands(bits, 3)
    calls = s.calls()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for _, call in calls.values():
            call()
    torch.cuda.current_stream().wait_stream(side)
    graphs, got = [torch.cuda.CUDAGraph() for _ in range(2)], []
    for graph in graphs:
        with torch.cuda.graph(graph):
            got.append({k: call() for k, (_, call) in calls.items()})
    for turn in range(5):
        if turn > 1:
            for t in (s.q[0], s.v[1], s.S[0], s.P[1], s.state, s.x, s.rstd, s.dy, s.xhat, s.gamma[0], s.token[2][0], s.kw["decay"], s.active):
                t += 12345 + turn
        want = {k: tensors(call()) for k, (_, call) in calls.items()}
        for graph in graphs[::-1]:
            graph.replay()
        torch.cuda.synchronize()
        for out in got:
            for k in calls:
                assert all(torch.equal(a, b) for a, b in zip(tensors(out[k]), want[k])), (turn, k)
