"""How many rows a workgroup of a rotation takes, by the work of a row and their number, on devices that need not be there; turns scaled by the pair's number."""
import math

import pytest

from paper_2602_17698_amd import binding as sb
from recording_runtime import record

SCRIPT = r"""
import ctypes as C
def rows(tokens, heads, dim, dims, ld=0, cus=256):
    device(cus, 1)
    ctx = sb.Context(0, 0)
    A = fake(1)
    turns = sb.Rotary(A, dims // 2, 0, 1.0)
    ld = ld or heads * dim
    log()
    assert sb.load().sbits_rotate(ctx.h, C.addressof(turns), A, tokens, heads, dim, A, ld, dim, 1, 0, A, ld, dim) == 0
    line, = [x.split() for x in log() if x.startswith("launch")]
    return "rows" in line[1], int(line[3].split(",")[0])
answer([rows(*a) for a in %r])
"""


def test_rows_of_a_workgroup(tmp_path):
    cases = [
        ((100000, 1, 64, 64), 64),             # 4 pieces a row: all of 256 threads
        ((100000, 2, 64, 64), 32), ((100000, 1, 128, 128), 32), ((1000000, 1, 32, 32), 128), ((1000000, 1, 32, 16), 85),
        ((100000, 1, 256, 256), 16),           # 2048 angles
        ((100000, 1, 96, 16), 23),             # 1 piece of 8 pairs and 10 of 8 elements
        ((100000, 1, 64, 64, 65), 8),          # not aligned: a pair a thread
        ((8192, 40, 128, 128), 1), ((8192, 32, 64, 64), 2), ((8192, 33, 64, 64), 1),
        ((1, 1, 64, 64), 1), ((1023, 1, 64, 64), 1), ((1024, 1, 64, 64), 2), ((5000, 1, 64, 64), 9),   # two workgroups a CU
        ((5000, 1, 64, 64, 0, 32), 64)]
    for (case, want), (several, grid) in zip(cases, record(tmp_path, SCRIPT % [c for c, _ in cases])):
        assert several == (want > 1) and grid == -(-case[0] // want), (case, grid)


@pytest.mark.parametrize("context", [1, 3, 6, 7, 20, 150, 4096, 1e6, 1e12, 1e30])
@pytest.mark.parametrize("dims,base", [(64, 10000.0), (2, 10000.0), (128, 500000.0)])
def test_turns_by_the_pairs_number(context, dims, base):
    """Contexts so short that no pair turns once, or none 32 times, and so long that all do."""
    pairs, factor = dims // 2, 8.0
    got = sb.rotary_turns(dims, base, sb.ROTARY_INDEX, factor=factor, low=1.0, high=32.0, context=context)
    index = lambda n: pairs * math.log(context / (2 * math.pi * n)) / math.log(base)  # noqa: E731
    first, last = max(0, math.floor(index(32.0))), min(2 * pairs - 1, math.ceil(index(1.0)))
    for i, turns in enumerate(got):
        f = base ** (-i / pairs) / (2 * math.pi)
        want = f / factor if i >= last else f if i <= first else f * (last - i) / (last - first) + f / factor * (i - first) / (last - first)
        assert abs(turns - want) <= 1e-12 * f, (i, turns / f)
