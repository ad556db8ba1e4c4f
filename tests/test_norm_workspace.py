"""One workspace, sized for the largest batch, does for the norm's gradient of every smaller one.  The queries touch no GPU."""
import pytest

from paper_2402_02320_amd import spin

# around the numbers at which another count of waves a row, of rows a group or of groups begins
ROWS = sorted({r + d for r in (1, 4, 8, 255, 256, 257, 1024, 2048, 4096, 4100, 8192, 100000) for d in (-1, 0, 1, 2, 3)} - {0})


@pytest.mark.parametrize("ring", [spin, spin.ring32])
@pytest.mark.parametrize("dim", [1, 7, 255, 256, 257, 500, 1023, 1024, 1025, 2048, 4097, 8192])
def test_fewer_rows_never_need_more(dim, ring):
    for n in (1, 2, 3, 8):
        sizes = [ring.layernorm_grad_workspace_bytes(n, rows, dim) for rows in ROWS]
        assert sizes[0] > 0 and sizes == sorted(sizes), (n, list(zip(ROWS, sizes)))


@pytest.mark.parametrize("ring", [spin, spin.ring32])
def test_fewer_parties_never_need_more(ring):
    for rows, dim in ((3, 40), (5000, 256), (1029, 300), (515, 2049)):
        sizes = [ring.layernorm_grad_workspace_bytes(n, rows, dim) for n in range(1, 9)]
        assert sizes == sorted(sizes)
