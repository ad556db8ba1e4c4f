"""Results in place of operands, where that is allowed: the scores over C and the truncation tuple, the biased scores over x and the tuple."""
import pytest
import torch

from paper_2402_02320_amd import spin
from test_gpu_generation import BITS, RINGS, ints

pytestmark = pytest.mark.gpu


def words(bits, *shape):
    return torch.empty(shape, dtype=torch.int64 if bits == 64 else torch.int32, device="cuda").random_(-2 ** (bits - 1), 2 ** (bits - 1) - 1)


@BITS
@pytest.mark.parametrize("n,share,nodes,context", [(2, 1, 1, 300), (3, 2, 1, 95), (3, 4, 5, 200), (5, 1, 3, 130), (8, 2, 10, 70)])
def test_scores(bits, n, share, nodes, context):
    ring = RINGS[bits][0]
    torch.manual_seed(n + nodes)
    batch, kv, dim, columns = 2, 2, 64, context + nodes + 3
    pool, table = words(bits, n + 1, 50, kv, 16, dim), torch.randperm(50)[:2 * 22].view(2, 22).int().cuda()
    lead = (n, batch, kv * share, nodes)
    Q, A, tensors = words(bits, *lead, dim), words(bits, *lead, dim), [words(bits, *lead, columns) for _ in range(4)]
    lut, bias = spin.relative_buckets(32, 20, False).cuda(), words(bits, n, kv * share, 32)

    def call(C, r, top, msb, out=None):
        return ring.cache_scores(pool, table, ints([context, context // 3]), Q, A, C, f=9, tuple_=[r, top, msb], masked=-3, bias=(bias, lut), out=out)
    want = call(*tensors)
    for k in range(4):
        own = [t.clone() for t in tensors]
        assert call(*own, out=own[k]) is own[k] and torch.equal(own[k], want)
        assert all(torch.equal(a, b) for j, (a, b) in enumerate(zip(own, tensors)) if j != k)


@BITS
@pytest.mark.parametrize("n,Q,K", [(1, 1, 300), (3, 40, 41), (8, 9, 200), (3, 300, 1300)])
def test_biased_scores(bits, n, Q, K):
    ring = RINGS[bits][0]
    torch.manual_seed(n + Q)
    tensors = [words(bits, n, 2, 3, Q, K) for _ in range(4)]
    lut, bias = spin.relative_buckets(32, 20, True).cuda(), words(bits, n, 3, 32)

    def call(x, r, top, msb, out=None):
        return ring.relbias_trunc(x, bias, lut, f=9, tuple_=[r, top, msb], causal=True, first=K - Q, lengths=ints([K, K // 2]), masked=-3, out=out)
    want = call(*tensors)
    for k in range(4):
        own = [t.clone() for t in tensors]
        assert call(*own, out=own[k]) is own[k] and torch.equal(own[k], want)
        assert all(torch.equal(a, b) for j, (a, b) in enumerate(zip(own, tensors)) if j != k)
