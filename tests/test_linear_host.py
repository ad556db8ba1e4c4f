"""Host code of the calls of linear attention and layer norm in a separate program under AddressSanitizer and UndefinedBehaviorSanitizer."""
import os

from test_generation_host import build_and_run
from test_sanitizers import SAN


def test_numbers_and_refusals(tmp_path):
    from paper_2402_02320_amd import build
    build_and_run(tmp_path, os.path.join(build.CSRC, "linear_api.hip"), os.path.join(SAN, "linear_san.hip"))
