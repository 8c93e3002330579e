"""Products with the most rows of W, or of x, that are accepted: every launch has fewer than 2^32 threads along an axis and 65536 workgroups along the other, and
the launches together cover all rows."""
from recording_runtime import record
from test_mx_grids import launches

SCRIPT = r"""
import ctypes as C
ctx = sb.Context(0, 0)
lib = sb.load()
def mx(rows, cols):
    return sb.Mx(fake(rows * cols // 2), fake(rows * sb.mx_scale_pitch(cols)), rows, cols, cols // 2, sb.mx_scale_pitch(cols))
many = (1 << 31) - 1
out = {}
log()
def call(name, what, *args):
    rc = getattr(lib, "sbits_" + what)(ctx.h, *[C.addressof(a) if isinstance(a, C.Structure) else a for a in args])
    out[name] = [rc, [line for line in log() if line.startswith("launch")]]
for batch in (1, 40):
    w = mx(many, 32)
    call("product %d" % batch, "mx_gemm", w, fake(batch * 64), 32, None, batch, 0, fake(many * batch * 4), 0, 1 << 31, None, 0)
    w = mx(many - 1, 32)
    call("gated %d" % batch, "mx_gemm", w, fake(batch * 64), 32, None, batch, 1, fake(many * batch * 4), 0, 1 << 31, None, 0)
call("rows of x", "mx_gemm", mx(8, 32), fake(many * 64), 32, None, many, 0, fake(many * 32), 0, 8, None, 0)
answer(out)
"""


def test_launches_of_products_of_the_largest_sizes(tmp_path):
    many = 2 ** 31 - 1
    seen = record(tmp_path, SCRIPT)
    for name, (rc, lines) in seen.items():
        assert rc == 0 and lines, name
        for grid, block in launches(lines):
            assert grid[0] * block < 2 ** 32 and grid[1] < 65536, (name, grid, block)
    for name, outs, x_tiles in (("product 1", many, 1), ("product 40", many, 3), ("gated 1", many // 2, 1), ("gated 40", many // 2, 3)):
        grids = launches(seen[name][1])
        # 64 rows of W to a workgroup
        assert all(g[1] == x_tiles for g, _ in grids) and sum(g[0] for g, _ in grids) == -(-outs // (32 if "gated" in name else 64)), (name, grids[:3])
    assert sum(g[1] for g, _ in launches(seen["rows of x"][1])) == -(-many // 16)
