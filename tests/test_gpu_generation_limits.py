"""As many sequences as a launch grid's third axis holds, with the parties apart on it (f = 0) and together."""
import pytest
import torch

from test_gpu_generation import RINGS, ints

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("bits", [64, 32])
@pytest.mark.parametrize("n,batch,share", [(8, 8191, 1), (8, 8191, 5), (1, 65535, 1)])
def test_as_many_sequences_as_there_may_be(bits, n, batch, share):
    ring, _, _ = RINGS[bits]
    word = torch.int64 if bits == 64 else torch.int32
    torch.manual_seed(batch + share)

    def u(*shape):
        return torch.empty(shape, dtype=word, device="cuda").random_(-2 ** (bits - 1), 2 ** (bits - 1) - 1)
    dim, context = 8, 4
    columns = context + 1
    pool = u(n + 1, 7, 1, 16, dim)
    table = ints([[k % 7] for k in range(batch)])
    contexts = ints([context] * batch)
    rows = pool[:, table[:, 0].long(), 0, :columns]            # [slots, batch, columns, dim]
    Q, A, C = u(n, batch, share, 1, dim), u(n, batch, share, 1, dim), u(n, batch, share, 1, columns)
    E = (Q - A).sum(0, dtype=word)
    want = C + ((E[None, :, :, 0, None] * rows[1:, :, None]).sum(-1, dtype=word) + (A[:, :, :, 0, None] * rows[0][None, :, None]).sum(-1, dtype=word))[:, :, :, None]
    assert torch.equal(ring.cache_scores(pool, table, contexts, Q, A, C), want)
    P, A, C = u(n, batch, share, 1, columns), u(n, batch, share, 1, columns), u(n, batch, share, 1, dim)
    E = (P - A).sum(0, dtype=word)
    want = C + ((E[None, :, :, 0, :, None] * rows[1:, :, None]).sum(-2, dtype=word) + (A[:, :, :, 0, :, None] * rows[0][None, :, None]).sum(-2, dtype=word))[:, :, :, None]
    assert torch.equal(ring.cache_values(pool, table, contexts, P, A, C), want)


def test_join_of_more_elements_than_one_axis_holds():
    """2^30 words of a result that is summed in two ranges, against the same call by quarters of the batch."""
    n, batch, heads, nodes, dim, columns = 8, 1024, 8, 64, 256, 521
    if torch.cuda.mem_get_info()[0] < 80 << 30:
        pytest.skip("needs 80 GB")
    ring = RINGS[32][0]
    torch.manual_seed(3)

    def u(*shape):
        return torch.empty(shape, dtype=torch.int32, device="cuda").random_(-2 ** 31, 2 ** 31 - 1)
    pool, table = u(n + 1, 9, 2, 128, dim), torch.stack([torch.randperm(9)[:5] for _ in range(batch)]).int().cuda()
    contexts = ints([(457 + 31 * k) % 458 for k in range(batch)])
    P, A, C = u(n, batch, heads, nodes, columns), u(n, batch, heads, nodes, columns), u(n, batch, heads, nodes, dim)
    size = ring.cache_values_workspace_bytes(pool, table, heads, nodes, columns)
    assert C.numel() >= 1 << 30 and size > 8 * C.numel()
    got = ring.cache_values(pool, table, contexts, P, A, C)
    for k in range(0, batch, 256):
        part = slice(k, k + 256)
        want = ring.cache_values(pool, table[part].contiguous(), contexts[part].contiguous(), *[t[:, part].contiguous() for t in (P, A, C)])
        assert torch.equal(got[:, part], want)
    del P, A, C, got, want
    torch.cuda.empty_cache()
