"""The rules that say how many waves a row of the norm has, and how many rows a wave or workgroup of its gradient, against what the cases of tests/test_gpu_norm_rows.py are there
for: another rule would take them out of the tests unseen.  Compiled for the host, nothing runs."""
import os
import subprocess

import pytest

from test_gpu_norm_rows import FOUR_WAVES, SEVERAL_ROWS

SOURCE = """#include "layernorm_grad.hip"
using namespace spin;
constexpr int words(int rows, int dim)
{
    int each = 0;
    for_dim(rows, dim, [&](auto, auto e) { each = decltype(e)::value; });
    return each;
}
"""


def claims():
    for n, rows, dim, _ in FOUR_WAVES.values():
        yield "norm_waves(%d, %d) == 4" % (rows, dim)
    for (n, rows, dim, _), (waves, each, run), lean in SEVERAL_ROWS.values():
        yield "norm_waves(%d, %d) == %d && words(%d, %d) == %d" % (rows, dim, waves, rows, dim, each)
        yield "norm_runs(%d, %d).run == %d" % (rows, dim, run)
        # the last group has fewer rows than the others
        yield "norm_runs({0}, {1}).groups * norm_runs({0}, {1}).run * norm_rows_at_once({0}, {1}) > {0}".format(rows, dim)
        for word, own in zip(("u64", "u32"), lean):
            yield "kLean<%d, %s, %d, %d> == %s" % (n, word, waves, each, str(own).lower())


def compiled(tmp_path, lines, more=""):
    from paper_2402_02320_amd import build
    if not os.path.exists(build.hipcc()):
        pytest.skip("hipcc not available")
    source = tmp_path / "rows.hip"
    source.write_text(SOURCE + more + "".join('static_assert(%s, "");\n' % c for c in lines))
    return subprocess.run([build.hipcc()] + build.COMPILE_FLAGS + ["--cuda-host-only", "-fsyntax-only", "-fconstexpr-steps=10000000", "-I", build.CSRC, str(source)], stdout=subprocess.PIPE,
                          stderr=subprocess.STDOUT, text=True)


def test_the_cases_are_what_they_say(tmp_path):
    res = compiled(tmp_path, claims())
    assert res.returncode == 0, res.stdout[-4000:]


def test_another_rule_would_be_seen(tmp_path):
    assert "static assertion failed" in compiled(tmp_path, ["norm_waves(300, 333) == 16"]).stdout


ROOM = """constexpr bool room(int dim)
{
    for (int rows = 1; rows < 9000; ++rows) {
        const NormRuns r = norm_runs(rows, dim);
        if (r.groups > norm_most_groups(rows, dim) || (long)r.groups * r.run * norm_rows_at_once(rows, dim) < rows || norm_most_groups(rows, dim) > norm_most_groups(rows + 1, dim)) return false;
    }
    return true;
}
"""


def test_at_least_as_many_groups_have_room(tmp_path):
    res = compiled(tmp_path, ["room(%d)" % dim for dim in (1, 256, 257, 1024, 1025, 8192)], ROOM)
    assert res.returncode == 0, res.stdout[-4000:]
