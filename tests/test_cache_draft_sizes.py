"""Drafts of sizes that there are not, on the CPU."""
import pytest

from paper_2402_02320_amd import spin
from test_cache_pages import Model, calls_of_the_oracle  # noqa: F401 - the calls' fixture


def test_a_draft_of_less_than_no_rows_is_refused():
    m = Model(4)
    a = m.add()
    m.append([a], [5])
    with pytest.raises(spin.SpinError):
        m.cache.keep([a], -3, [[]])
    m.check()
    m.keep([a], 0, [[]])
    m.keep([a], 5, [[]])
    m.check()
