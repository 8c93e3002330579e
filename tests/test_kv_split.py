"""How the attention's kernels divide up their work, in arithmetic that the host can run."""
import random
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


# ---- few rows' keys, shared out ------------------------------------------------------------------------
WALK = r"""
#include <vector>
// a batch: kv_heads, workgroups at most, space for parts, rows announced, sequences (rows, tiles of keys); for each workgroup its pieces of items, with a slot or -1, then for each item the
// slots that the join reads
int main()
{
    int kv, most, space, announced, n;
    while (scanf("%d %d %d %d %d", &kv, &most, &space, &announced, &n) == 5) {
        std::vector<int> rows(n), keys(n), tiles(n);
        std::vector<int64_t> begin(n + 1, 0);
        for (int b = 0; b < n; ++b) {
            if (scanf("%d %d", &rows[b], &keys[b]) != 2) return 1;
            tiles[b] = (rows[b] + 15) / 16;
            begin[b + 1] = begin[b] + (int64_t)tiles[b] * kv * keys[b];
        }
        const int64_t total = begin[n];
        const int workgroups = few_workgroups(most, space, total);
        int at, item, off;
        auto cuttable = [&](int b) { return few_cuttable(space, announced, rows[b], keys[b]); };
        auto cut = [&](int w) {
            if (w == workgroups) return total;
            const int64_t x = few_cut(w, workgroups, total);
            for (at = 0; begin[at + 1] <= x;) ++at;
            item = (int)((x - begin[at]) / keys[at]);
            const int in = (int)(x - begin[at] - (int64_t)item * keys[at]);
            off = few_snap(cuttable(at), keys[at], in);
            return x + off - in;
        };
        for (int w = 0; total && w < workgroups; ++w) {
            const int64_t stop = cut(w + 1), from = cut(w);
            int64_t left = stop - from;
            if (left < 0) return 2;
            for (; left > 0; ++item, off = 0) {
                if (off == keys[at]) continue;
                while (item >= tiles[at] * kv) for (item = 0, ++at; tiles[at] == 0;) ++at;
                const int last = (int)(off + left < keys[at] ? off + left : keys[at]);
                left -= last - off;
                printf("piece %d %d %d %d %d ", at, item, off, last, off == 0 && last == keys[at] ? -1 : 2 * w + (off == 0));
            }
        }
        for (int b = 0; b < n; ++b)
            for (int i = 0; i < tiles[b] * kv && cuttable(b); ++i) {
                const FewCuts c = few_cuts(begin[b] + (int64_t)i * keys[b], keys[b], workgroups, total);
                if (c.past > c.first) printf("join %d %d %d %d 0 ", b, i, c.first, c.past);
            }
        printf("\n");
    }
}
"""


def test_every_tile_of_keys_once_and_the_join_reads_what_was_written(tmp_path):
    exe = compiled(tmp_path, WALK)
    rng = random.Random(3)
    cases = []
    for _ in range(4000):
        n = rng.choice([1, 1, 2, 3, 10, 70, 150])
        long = rng.choice([1, 1, 1, 1000])
        cases.append([rng.choice([1, 2, 5, 8]), rng.choice([1, 2, 3, 17, 64, 256, 512]), rng.choice([0, 1, 1]), rng.choice([1, 4, 16, 64]), n]
                     + [x for _ in range(n) for x in (rng.choice([0, 1, 4, 16, 17, 40, 64, 100]), rng.choice([1, 2, 5, 16, 17, 20, 41, 300]) * rng.choice([1, long]))])
    out = subprocess.run([exe], input="\n".join(" ".join(map(str, c)) for c in cases), stdout=subprocess.PIPE, text=True, check=True).stdout.split("\n")[:-1]
    cuts = 0
    for c, line in zip(cases, out):
        kv, most, space, announced, n = c[:5]
        rows, keys = c[5::2], c[6::2]
        words = line.split()
        taken, slots, read = {}, {}, {}
        for i in range(0, len(words), 6):
            kind, (b, item, first, last, slot) = words[i], map(int, words[i + 1:i + 6])
            if kind == "piece":
                taken.setdefault((b, item), []).append((first, last))
                if slot >= 0:
                    assert space and keys[b] > 16 and rows[b] <= announced and slot < 2 * most and slot not in slots
                    slots[slot] = (b, item, len(taken[b, item]) - 1)
            else:                                                # its first part is workgroup first - 1's, the others begin at the cuts
                for part, s in enumerate([2 * (first - 1) + 1] + [2 * w for w in range(first, last)]):
                    assert s not in read
                    read[s] = (b, item, part)
        assert slots == read
        cuts += len(slots)
        for b in range(n):
            for item in range(-(-rows[b] // 16) * kv):
                pieces = taken.pop((b, item))
                assert pieces[0][0] == 0 and pieces[-1][1] == keys[b] and all(x[1] == y[0] for x, y in zip(pieces, pieces[1:]))
        assert not taken
    assert cuts > 10000
