"""Calls with more sequences, heads or parties than a launch grid's second and third axes hold, on the CPU: refused before anything is launched, so the
pointers are never followed."""
import pytest

from paper_2402_02320_amd import spin
from test_generation_arguments import ERANGE, P, cache

L = pytest.fixture(scope="module")(lambda: spin.lib())


@pytest.mark.parametrize("pre", ["spin_", "spin32_"])
@pytest.mark.parametrize("n,batch", [(8, 8192), (2, 32768), (8, 65535)])
def test_parties_apart_on_one_axis(L, pre, n, batch):
    """Without truncation a workgroup has one party."""
    c = cache(n=n, heads=1, batch=batch, K=P, V=P)
    assert getattr(L, pre + "cache_scores")(c, 1, 1, 40, 0, P, None, P, P, P, None, None, None, 5, None, None, P, None) == ERANGE
    assert getattr(L, pre + "cache_values")(c, 1, 1, 40, 0, P, None, P, P, P, None, None, None, P, P, 1 << 40, None) == ERANGE
    # by digits too
    assert getattr(L, pre + "cache_scores")(c, 7, 3, 40, 0, P, None, P, P, P, None, None, None, 5, None, None, P, None) == ERANGE
    assert getattr(L, pre + "cache_values")(c, 7, 3, 40, 0, P, None, P, P, P, None, None, None, P, P, 1 << 40, None) == ERANGE


@pytest.mark.parametrize("heads,dim", [(32768, 256), (65535, 136)])
def test_column_blocks_and_heads_on_one_axis(L, heads, dim):
    """Of 64-bit words a row longer than 128 takes two blocks of columns (one row a cached head; more rows are fewer heads)."""
    c = cache(n=1, pages=1, heads=heads, dim=dim, batch=1)
    assert L.spin_cache_values(c, heads, 1, 40, 9, P, None, P, P, P, P, P, P, P, P, 1 << 40, None) == ERANGE
