"""Layer norm on shares, forward and backward, word for word against the numpy oracle."""
import numpy as np
import pytest
import torch

from oracle import linear as lin
from test_gpu_generation import BITS, RINGS, same, uniform
from test_gpu_linattn import all_same, on

pytestmark = pytest.mark.gpu

# name: n, rows, dim, iterations
CASES = {
    "one_word": (3, 1, 1, 0),
    "one_row": (3, 1, 1024, 6),
    "two_wide_rows": (2, 2, 8192, 3),
    "odd": (2, 37, 333, 5),
    "narrow": (3, 300, 7, 2),
    "one_party": (1, 5, 64, 1),
    "eight_parties": (8, 9, 500, 4),
    "eight_wide": (8, 3, 4100, 2),
    "five_parties": (5, 50, 257, 3),
    "many_rows": (2, 2500, 48, 2),
    "below_a_wave": (4, 3, 63, 16),
    "long_odd": (3, 11, 2049, 2),
    "six": (6, 4, 1025, 1),
    "seven": (7, 4, 129, 1),
}


def numbers(bits):
    """f, shift, (offset, slope), eps"""
    return (16, 26, (3 << 15, 1 << 14), 1) if bits == 64 else (9, 15, (3 << 8, 1 << 7), 1)


def forward(name, bits):
    n, rows, dim, iterations = CASES[name]
    rng = np.random.default_rng(sum(map(ord, name)))

    def u(*shape):
        return uniform(rng, bits, n, *shape)
    f, shift, line, eps = numbers(bits)
    return (u(rows, dim), (u(dim), u(dim)), u(dim), (u(rows, dim), u(rows, dim)), (u(rows, dim), u(rows, dim)),
            ([u(rows, dim) for _ in range(3)], [u(rows, dim) for _ in range(3)]), u(15 * (iterations + 1), rows)), (f, shift, line, eps)


def backward(name, bits):
    n, rows, dim, _ = CASES[name]
    rng = np.random.default_rng(1 + sum(map(ord, name)))

    def u(*shape):
        return uniform(rng, bits, n, *shape)
    f, shift, _, _ = numbers(bits)
    return (u(rows, dim), u(rows, dim), u(rows), (u(dim), u(dim)), [u(rows, dim) for _ in range(3)], (u(rows, dim), u(rows, dim)),
            ([u(rows, dim) for _ in range(3)], [u(rows, dim) for _ in range(3)]), u(22, rows), u(4, dim)), (f, shift)


@BITS
@pytest.mark.parametrize("name", sorted(CASES))
def test_forward(name, bits):
    args, more = forward(name, bits)
    ring, want, ops = RINGS[bits][0], lin.layernorm(*args, *more), on(args)
    assert all_same(ring.layernorm(*ops, *more), want)
    got = ring.layernorm(*ops, *more, out=(torch.empty_like(ops[0]), None, None))
    assert same(got[0], want[0]) and got[1] is None and got[2] is None
    rstd = torch.empty_like(ops[0][:, :, 0])
    assert all_same(ring.layernorm(*ops, *more, out=(ops[4][1], ops[5][0][0], rstd)), want)               # in place of C2 and of t1's r


@BITS
@pytest.mark.parametrize("name", sorted(CASES))
def test_backward(name, bits):
    args, more = backward(name, bits)
    ring, want, ops = RINGS[bits][0], lin.layernorm_grad(*args, *more), on(args)
    assert all_same(ring.layernorm_grad(*ops, *more), want)
    need = ring.layernorm_grad_workspace_bytes(*ops[0].shape)
    ws = torch.full((need + 512,), 0x5A, dtype=torch.uint8, device="cuda")
    dgamma, dbeta = torch.empty_like(ops[3][0]), torch.empty_like(ops[3][0])
    assert all_same(ring.layernorm_grad(*ops, *more, out=(ops[6][1][1], dgamma, dbeta), workspace=ws[:need]), want)       # in place of t2's r_top
    assert bool((ws[need:] == 0x5A).all())
