"""Linear attention and layer norm on tensors of more than 2^32 words, a party's share more than 2^31: their ends word for word against the numpy oracle.  Two tensors of
random words stand for all operands of that size."""
import numpy as np
import pytest
import torch

from oracle import linear as lin
from oracle.generation import trunc
from test_gpu_generation import RINGS, same

pytestmark = pytest.mark.gpu
WORDS = 2 ** 31 + 2 ** 20                  # of a party's share, at least what the calls below take
NUMPY = {64: np.uint64, 32: np.uint32}


class Big:
    def __init__(self, bits):
        torch.manual_seed(bits)
        kind = torch.int64 if bits == 64 else torch.int32
        self.ring, self.bits = RINGS[bits][0], bits
        self.words = [torch.empty(2 * WORDS, dtype=kind, device="cuda").random_(-2 ** (bits - 1), 2 ** (bits - 1) - 1) for _ in range(2)]

    def of(self, which, *shape):
        return self.words[which][:int(np.prod(shape))].view(shape)


@pytest.fixture(scope="module", params=[32, 64])
def big(request):
    torch.cuda.empty_cache()
    yield Big(request.param)
    torch.cuda.empty_cache()


def host(v):
    """Of a tensor, or of the tensors in tuples and lists, the words in numpy."""
    if isinstance(v, torch.Tensor):
        return v.cpu().numpy().view(NUMPY[8 * v.element_size()])
    return type(v)(host(k) for k in v)


def ends(v, axis, last):
    if isinstance(v, torch.Tensor):
        return v.narrow(axis, v.shape[axis] - last, last)
    return type(v)(ends(k, axis, last) for k in v)


def check_size(t):
    assert t[0].numel() > 2 ** 31 and t.numel() > 2 ** 32


TOKENS, CHUNK = 2 ** 23 + 77, 32
CHUNKS, TAIL = -(-TOKENS // CHUNK), 2      # checked chunks, the last one cut
TAIL_TOKENS = TOKENS - (CHUNKS - TAIL) * CHUNK


def test_scores(big):
    x, y = [(big.of(k, 2, 1, 1, TOKENS, 256), big.of(1 - k, 2, 1, 1, TOKENS, 256)) for k in range(2)]
    check_size(x[0])
    C, t = big.of(0, 2, 1, 1, CHUNKS, CHUNK, CHUNK), [big.of(k % 2, 2, 1, 1, CHUNKS, CHUNK, CHUNK) for k in range(3)]
    got = big.ring.linattn_scores(x, y, C, t, 9)
    want = lin.scores(*[host(ends(v, 3, TAIL_TOKENS)) for v in (x, y)], *[host(ends(v, 3, TAIL)) for v in (C, t)], 9)
    assert same(ends(got, 3, TAIL).contiguous(), want)


@pytest.mark.parametrize("reverse", [False, True])
def test_outputs(big, reverse):
    y, C = (big.of(0, 2, 1, 1, TOKENS, 256), big.of(1, 2, 1, 1, TOKENS, 256)), big.of(0, 2, 1, 1, TOKENS, 256)
    check_size(C)
    t = [big.of((1 + k) % 2, *C.shape) for k in range(3)]
    P, x, S = [(big.of(1, 2, 1, 1, *shape), big.of(0, 2, 1, 1, *shape)) for shape in ((CHUNKS, CHUNK, CHUNK), (TOKENS, 8), (CHUNKS, 8, 256))]
    got = big.ring.linattn_outputs(P, y, x, S, C, t, 9, reverse=reverse)
    chunks, tokens = [host(ends(v, 3, TAIL)) for v in (P, S)], [host(ends(v, 3, TAIL_TOKENS)) for v in (y, x, C, t)]
    want = lin.outputs(chunks[0], tokens[0], tokens[1], chunks[1], tokens[2], tokens[3], 9, reverse=reverse)
    assert same(ends(got, 3, TAIL_TOKENS).contiguous(), want)


def test_states(big):
    chunks = 2 ** 15 + 7
    x, y = [(big.of(k, 2, 1, 1, chunks * CHUNK, 256), big.of(1 - k, 2, 1, 1, chunks * CHUNK, 256)) for k in range(2)]
    C, t = big.of(0, 2, 1, 1, chunks, 256, 256), [big.of(k % 2, 2, 1, 1, chunks, 256, 256) for k in range(3)]
    check_size(C)
    got, last = big.ring.linattn_states(x, y, C, t, 9, CHUNK)
    at = host(got[:, :, :, -TAIL - 1])     # from a state of the result to the end
    want, end = lin.states(*[host(ends(v, 3, (TAIL + 1) * CHUNK)) for v in (x, y)], *[host(ends(v, 3, TAIL + 1)) for v in (C, t)], 9, CHUNK, first=at)
    assert same(ends(got, 3, TAIL).contiguous(), want[:, :, :, 1:]) and same(last, end)


def test_step(big):
    batch = 2 ** 15 + 9
    S, mask, C = big.of(0, 2, batch, 1, 256, 256), big.of(1, 2, batch, 1, 256, 256), big.of(0, 2, batch, 1, 256, 256)
    check_size(S)
    tS = [big.of((1 + k) % 2, *S.shape) for k in range(3)]
    vectors = [(big.of(k, 2, batch, 1, 256), big.of(1 - k, 2, batch, 1, 256)) for k in (0, 1, 0)]
    CO, tO = big.of(1, 2, batch, 1, 256), [big.of(k % 2, 2, batch, 1, 256) for k in range(3)]
    got = big.ring.linattn_step(S, *vectors, mask, (C, CO), (tS, tO), 9)
    want = lin.step(*[host(ends(v, 1, 2)) for v in (S, *vectors, mask)], host(ends((C, CO), 1, 2)), host(ends((tS, tO), 1, 2)), 9)
    assert all(same(ends(g, 1, 2).contiguous(), w) for g, w in zip(got, want))


ROWS, DIM = 2 ** 20 + 3, 2048


def test_norm(big):
    x = big.of(0, 2, ROWS, DIM)
    check_size(x)
    masks, C = (big.of(1, *x.shape), x), (big.of(1, *x.shape), x)
    tuples = tuple([big.of((j + k) % 2, *x.shape) for k in range(3)] for j in range(2))
    gamma, beta, words = (big.of(0, 2, DIM), big.of(1, 2, DIM)), big.of(1, 2, DIM), big.of(1, 2, 30, ROWS)
    got = big.ring.layernorm(x, gamma, beta, masks, C, tuples, words, 9, 15, (768, 128), 1)
    want = lin.layernorm(host(ends(x, 1, 2)), host(gamma), host(beta), *[host(ends(v, 1, 2)) for v in (masks, C, tuples)], host(ends(words, 2, 2)), 9, 15, (768, 128), 1)
    assert all(same(ends(g, 1, 2).contiguous(), w) for g, w in zip(got, want))


def test_norm_grad(big):
    dy, xhat = big.of(0, 2, ROWS, DIM), big.of(1, 2, ROWS, DIM)
    check_size(dy)
    masks, C = (xhat, dy, xhat), (dy, xhat)
    tuples = tuple([big.of((j + k) % 2, *dy.shape) for k in range(3)] for j in range(2))
    gamma, rstd, words, columns = (big.of(0, 2, DIM), big.of(1, 2, DIM)), big.of(0, 2, ROWS), big.of(1, 2, 22, ROWS), big.of(0, 2, 4, DIM)
    dx, dgamma, dbeta = big.ring.layernorm_grad(dy, xhat, rstd, gamma, masks, C, tuples, words, columns, 9, 15)
    want = lin.layernorm_grad(*[host(ends(v, 1, 2)) for v in (dy, xhat, rstd)], host(gamma), *[host(ends(v, 1, 2)) for v in (masks, C, tuples)], host(ends(words, 2, 2)),
                              host(columns), 9, 15)
    assert same(ends(dx, 1, 2).contiguous(), want[0])
    z, sums = torch.zeros_like(dgamma), torch.zeros_like(dbeta)
    for a, b in zip(dy.split(2 ** 15, 1), xhat.split(2 ** 15, 1)):        # dy is opened against xhat, and xhat against dy
        e = (a - b).sum(0, dtype=a.dtype)
        z += (b * -e + e * a).sum(1, dtype=a.dtype)
        z[0] -= (e * e).sum(0, dtype=a.dtype)
        sums += a.sum(1, dtype=a.dtype)
    w = host(columns)
    assert same(dbeta, host(sums)) and same(dgamma, trunc(w[:, 0] + host(z), [np.ascontiguousarray(w[:, 1 + k]) for k in range(3)], 9))
