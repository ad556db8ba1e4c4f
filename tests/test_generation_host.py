"""Host code of the cache, attention and bias calls in separate programs under AddressSanitizer and UndefinedBehaviorSanitizer."""
import os
import subprocess

import pytest

from test_sanitizers import ROOT, SAN, run


def build_and_run(tmp_path, *sources):
    from paper_2402_02320_amd import build
    hipcc = build.hipcc()
    if not os.path.exists(hipcc):
        pytest.skip("hipcc not available")
    host_san = ["-Xarch_host", "-fsanitize=address", "-Xarch_host", "-fsanitize=undefined", "-Xarch_host", "-fno-sanitize-recover=all"]
    quiet = dict(stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True, cwd=ROOT)
    objects = []
    for source in sources:
        objects.append(str(tmp_path / (os.path.basename(source) + ".o")))
        res = subprocess.run([hipcc] + build.COMPILE_FLAGS + ["-O1", "-g"] + host_san + ["-c", source, "-o", objects[-1]], **quiet)
        assert res.returncode == 0, res.stdout[-3000:]
    exe = str(tmp_path / "program")
    res = subprocess.run([hipcc, "--offload-arch=gfx950", "-Wno-unused-command-line-argument"] + host_san[:4] + objects + ["-o", exe], **quiet)
    assert res.returncode == 0, res.stdout[-3000:]
    run(exe)


def test_rows_of_a_diagonal(tmp_path):
    build_and_run(tmp_path, os.path.join(SAN, "diagonal_san.hip"))


def test_grids(tmp_path):
    build_and_run(tmp_path, os.path.join(SAN, "grid_san.hip"))


def test_what_the_launchers_are_given(tmp_path):
    from paper_2402_02320_amd import build
    build_and_run(tmp_path, os.path.join(build.CSRC, "generation_api.hip"), os.path.join(SAN, "dispatch_san.hip"))
