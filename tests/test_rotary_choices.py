"""How many rows a workgroup of a rotation takes, by the work of a row and their number, on devices that need not be there."""
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
