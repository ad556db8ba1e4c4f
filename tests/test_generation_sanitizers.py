"""The host side of the paged cache's kernels under AddressSanitizer and UndefinedBehaviorSanitizer: index arithmetic over tables that hold anything,
and the entry points' argument checks (tests/sanitize/generation_san.hip).  A separate program, host code only."""
import os
import subprocess

import pytest

from test_sanitizers import ROOT, SAN, run


def test_indexes_and_argument_checks(tmp_path):
    from paper_2402_02320_amd import build
    hipcc = build.hipcc()
    if not os.path.exists(hipcc):
        pytest.skip("hipcc not available")
    host_san = ["-Xarch_host", "-fsanitize=address", "-Xarch_host", "-fsanitize=undefined", "-Xarch_host", "-fno-sanitize-recover=all"]
    obj_dir = os.path.join(os.path.dirname(build.LIB), "_build")
    others = [os.path.join(obj_dir, s.replace(".hip", ".o")) for s in build.SOURCES if s != "generation_api.hip"]
    if not all(os.path.exists(o) for o in others):
        build.build()
    objects = []
    for source in (os.path.join(build.CSRC, "generation_api.hip"), os.path.join(SAN, "generation_san.hip")):
        objects.append(str(tmp_path / (os.path.basename(source) + ".o")))
        res = subprocess.run([hipcc] + build.COMPILE_FLAGS + ["-O1", "-g"] + host_san + ["-c", source, "-o", objects[-1]],
                             stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True, cwd=ROOT)
        assert res.returncode == 0, res.stdout[-3000:]
    exe = str(tmp_path / "generation_san")
    res = subprocess.run([hipcc, "--offload-arch=gfx950", "-Wno-unused-command-line-argument"] + host_san[:4] + objects + others + ["-o", exe],
                         stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
    assert res.returncode == 0, res.stdout[-3000:]
    run(exe)
