"""examples/block.py: layer norm, attention over chunks, all gradients and tokens one at a time, run together; every stage against float64 from the opened values
that it was given, gradients against autograd's.

Errors are bounded by arithmetic.  u = 2^-16 is a unit of the fixed point; a truncation of less than 2^62 is off by less than one unit, and encodings do not count, since a stage is
given what was encoded.  A decay weight is off by at most e = 2^-21, 1 / dim by at most 2^-27, and max|.| is of the values at
hand."""
import importlib.util
import os

import pytest
import torch

pytestmark = pytest.mark.gpu
PATH = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "block.py")
U, E = 2.0 ** -16, 2.0 ** -21


@pytest.fixture(scope="module")
def example():
    spec = importlib.util.spec_from_file_location("block_example", PATH)
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


def top(x):
    return float(x.detach().abs().max())


def state_error(tokens, chunk, a, b):
    """S' = T(w S + sum w a (x) b): |S| and the sum are below tokens a b; roundings of earlier chunks are carried on with weights below 1."""
    return -(-tokens // chunk) * (2 * E * tokens * a * b + U)


def output_error(tokens, chunk, dim, p, y, x, s):
    """T(sum_j P_j y_j + w x . S), P = T(w p0 . p1), S a sum of s0 (x) s1."""
    return chunk * y * (E * dim * p[0] * p[1] + U) + dim * x * (state_error(tokens, chunk, *s) + E * tokens * s[0] * s[1]) + U


class NormError:
    """Of the forward pass on rows of `dim`.  The mean m is off by em; the squares' sum, whose deviations sum to zero, by dim em^2; the variance v by ev; Newton's last step
    y (3 - v y^2) / 2 rounds y^2, v y^2 and its result, and earlier steps' errors enter squared (one unit more)."""

    def __init__(self, x, gamma):
        dim, c = x.shape[-1], x - x.mean(-1, keepdim=True)
        v = c.square().mean(-1)
        assert 0.4 < float(v.min()) and float(v.max()) < 2       # where six steps converge: 1.5 - v / 4 is off by at most 0.42, then 0.3, 0.12, 0.022, 7e-4, 8e-7, 1e-12
        self.m = dim * top(x) * 2.0 ** -27 + U
        ev = self.m ** 2 + U / dim + float(v.max()) * dim * 2.0 ** -27 + U
        self.r = 0.5 * float(v.min()) ** -1.5 * ev + U * (2 + 0.5 * float(v.max()) ** 0.5 + 0.5 * float(v.min()) ** -0.5)
        self.rstd = float(v.min()) ** -0.5
        self.xhat = top(c) * self.r + self.rstd * self.m + U
        self.y = top(gamma) * self.xhat + U


@pytest.mark.parametrize("n,heads,dim,chunk,lengths", [(3, 2, 32, 32, [70, 33]), (2, 3, 40, 64, [65, 130, 0]), (5, 1, 64, 128, [1, 100])])
def test_forward_backward_and_tokens(example, n, heads, dim, chunk, lengths):
    batch, tokens, width = len(lengths), max(lengths), heads * dim
    block = example.Block(n, batch, heads, dim, chunk)
    seen = block.seen
    _, state, kept = block.forward(block.shared("x", block.real(batch * tokens, width)), lengths)
    block.backward(block.shared("do", block.real(batch, heads, tokens, dim)), kept)

    def close(name, want, bound):
        assert top(seen[name] - want) <= bound, (name, top(seen[name] - want), bound)

    def leaves(*names):
        return [seen[k].clone().requires_grad_() for k in names]

    def check_projection():
        want = example.split(seen["y"] @ seen["weights"], batch, heads, dim)
        for name, t in zip("qkv", want):
            close(name, t.reshape(seen[name].shape), U + 1e-9)
    # the norm and its gradients
    x, gamma, beta = leaves("x", "gamma", "beta")
    y = example.norm(x, gamma, beta)
    error = NormError(x.detach(), gamma)
    close("y", y, error.y)
    (y * seen["dy"]).sum().backward()
    g, r, h = top(seen["dy"]) * top(gamma), error.rstd, top(seen["xhat"]) + error.xhat
    m1 = 2 * U + g * width * 2.0 ** -27                       # the mean of dy gamma
    m2 = U * h + g * error.xhat + U / width + g * h * width * 2.0 ** -27 + U                 # and of (dy gamma) xhat
    # dx = r (g - m1 - xhat m2), of which r, g, m1, xhat and m2 are off, and by r m1, r m2 (times xhat) and the whole, rounded
    close("dx", x.grad, error.r * (2 * g + g * h * h) + r * (U + m1 + h * m2 + error.xhat * g * h) + U * (2 + h))
    close("dgamma", gamma.grad, float(seen["dy"].abs().sum(0).max()) * error.xhat + U)
    close("dbeta", beta.grad, 1e-9)
    # the projection and its gradients
    check_projection()
    close("dweights", seen["y"].T @ seen["dqkv"], U + 1e-9)
    close("dy", seen["dqkv"] @ seen["weights"].T, U + 1e-9)
    # attention and its gradients
    q, k, v = leaves("q", "k", "v")
    o, S = example.attention(q, k, v, lengths)
    Q, K, V, D = top(q), top(k), top(v), top(seen["do"])
    close("o", o, output_error(tokens, chunk, dim, (Q, K), V, Q, (K, V)))
    close("last", S, state_error(tokens, chunk, K, V))
    (o * seen["do"]).sum().backward()
    close("dq", q.grad, output_error(tokens, chunk, dim, (D, V), K, D, (K, V)))
    close("dk", k.grad, output_error(tokens, chunk, dim, (D, V), Q, V, (Q, D)))
    close("dv", v.grad, output_error(tokens, chunk, dim, (Q, K), D, K, (Q, D)))
    # tokens one at a time, from the prompt's state; one sequence waits in the second step
    S = seen["last"]
    for step in range(3):
        active = [0 if step == 1 and b == 1 else 1 for b in range(batch)]
        _, state = block.token(block.shared("x", block.real(batch, width)), state, torch.tensor(active, dtype=torch.int32, device="cuda"))
        close("y", example.norm(*[seen[name] for name in ("x", "gamma", "beta")]), NormError(seen["x"], seen["gamma"]).y)
        check_projection()
        q, k, v = [seen[name][:, :, None] for name in "qkv"]
        o, S = example.attention(q, k, v, active, S)
        off = E * (top(S) + top(k) * top(v)) + U               # of a state's element, which the next step is given
        close("o", o[:, :, 0], dim * top(q) * off + U)
        close("last", S, off)
        S = seen["last"]


def test_a_prompt_is_its_tokens_one_at_a_time(example):
    """The last token's output and the state, by chunks and by single steps from nothing: both are within their bounds of one recurrence in float64."""
    n, heads, dim, chunk, tokens = 3, 2, 24, 32, 37
    block = example.Block(n, 1, heads, dim, chunk, seed=9)
    x = block.real(tokens, heads * dim)
    _, last, _ = block.forward(block.shared("x", x), [tokens])
    seen = dict(block.seen)
    state = torch.zeros_like(last)
    for t in range(tokens):
        _, state = block.token(block.shared("x", x[t:t + 1]), state)
    Q, K, V = top(seen["q"]) + 0.1, top(seen["k"]) + 0.1, top(seen["v"]) + 0.1
    # both have queries, keys and values off by two norms' errors times the weights' sums, and a rounding
    off = 2 * NormError(x, seen["gamma"]).y * float(seen["weights"].abs().sum(0).max()) + 2 * U
    assert off < 0.1
    of_state = state_error(tokens, chunk, K, V) + tokens * (2 * E * tokens * K * V + U) + tokens * off * (K + V)
    assert top(block.seen["last"] - seen["last"]) <= of_state
    of_output = output_error(tokens, chunk, dim, (Q, K), V, Q, (K, V)) + dim * (Q * of_state + off * tokens * K * V) + U
    assert top(block.seen["o"] - seen["o"][:, :, -1]) <= of_output
