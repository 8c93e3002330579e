"""How the attention's kernels divide up their work, in arithmetic that the host can run."""
import shutil
import subprocess

import pytest

from paper_2602_17698_amd import build


def compiled(path, main):
    cxx = shutil.which("g++")
    if cxx is None:
        pytest.skip("needs g++")
    (path / "main.cpp").write_text('#include <stdio.h>\n#include "kv_split.hpp"\nusing namespace sbits;\n' + main)
    exe = str(path / "split")
    subprocess.check_call([cxx, "-std=c++17", "-O1", "-Wall", "-Werror", "-I" + build.CSRC, str(path / "main.cpp"), "-o", exe])
    return exe


def run(exe, cases):
    out = subprocess.run([exe], input="\n".join(" ".join(map(str, c)) for c in cases), stdout=subprocess.PIPE, text=True, check=True).stdout
    return [tuple(map(int, line.split())) for line in out.split("\n")[:-1]]


LAST = (1 << 31) - 4096         # positions from here on are not there


@pytest.fixture(scope="module")
def keys(tmp_path_factory):
    return compiled(tmp_path_factory.mktemp("keys"), "int main() { int c, w, t, n, p; while (scanf(\"%d %d %d %d %d\", &c, &w, &t, &n, &p) == 5) {"
                    " const KeyRange r = seen_keys(c, w, t, n, p); printf(\"%d %d\\n\", r.first, r.last); } }\n")


def test_the_keys_that_a_row_sees(keys):
    cases = [(c, w, t, n, p) for c, windows in ((0, (0,)), (1, (0, 1, 3, 64, 1000))) for w in windows for t in (1, 8, 64, 70) for n in (0, 1, 5, 64, 70, 200)
             for p in (-70, -1, 0, 1, 7, 8, 63, 64, 65, 199) if p < max(n, 1)]
    for (c, w, t, n, p), (first, last) in zip(cases, run(keys, cases)):
        want = [k for k in range(min(n, t)) if not c or (k <= p and (not w or k > p - w))]
        assert list(range(first, last)) == want, (c, w, t, n, p)


def test_no_range_leaves_the_table(keys):
    """Rows whose window begins behind the last page of the table: their empty range is where the kernels end to look pages up."""
    sizes = (1, 8, 15, 64, 1000, 1 << 20, LAST)
    cases = [(c, w, t, n, p) for c, windows in ((0, (0,)), (1, (0, 1, 10, 5000, (1 << 31) - 1))) for w in windows for t in sizes for n in (0, *sizes, (1 << 31) - 1)
             for p in (-(1 << 31), -5000, -1, 0, n - 70, n - 1) if p < max(n, 1)]
    for case, (first, last) in zip(cases, run(keys, cases)):
        assert 0 <= first <= last <= case[2], case
