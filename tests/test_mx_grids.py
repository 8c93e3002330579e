"""The most rows and tokens that quantisation, routing and layers accept: every launch has fewer than 2^32 threads along an axis and 65536 workgroups along the others, and
the launches together cover all rows."""
import re

from recording_runtime import record

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
for experts in (1, 64, 512):
    r = sb.Router(experts, 1)
    call("route %d" % experts, "route", r, fake(many * experts * 4), 0, experts, None, many, fake(many * 4), fake(many * 4))
    call("gradient %d" % experts, "route_backward", r, fake(many * experts * 4), 0, experts, fake(many * 4), fake(many * 4), many, fake(many * experts * 4), experts)
call("quantise", "mx_quantize", fake(many * 64), 1, 32, mx(many, 32), None, 0)
r, tokens = sb.Router(2, 1), (1 << 30) - 1
up, down = mx(2 * 64, 32), mx(2 * 32, 32)
need = ctx.expert_layer_ws_bytes(r, tokens, up, down)
call("layer", "expert_layer", r, fake(tokens * 8), 0, 2, None, fake(tokens * 64), 32, tokens, up, down, fake(tokens * 64), 32, fake(tokens * 4), fake(tokens * 4), 0, fake(need), need)
answer(out)
"""


def launches(lines, kernel=""):
    """(grid, threads of a workgroup) of each."""
    found = [re.match(r"launch (\S+) grid (\d+),(\d+),(\d+) block (\d+)", line).groups() for line in lines]
    return [(tuple(int(v) for v in k[1:4]), int(k[4])) for k in found if kernel in k[0]]


def test_launches_of_the_largest_sizes(tmp_path):
    many = 2 ** 31 - 1
    seen = record(tmp_path, SCRIPT)
    for name, (rc, lines) in seen.items():
        assert rc == 0 and lines, name
        for grid, block in launches(lines):
            assert grid[0] * block < 2 ** 32 and grid[1] < 65536 and grid[2] < 65536, (name, grid, block)
    threads = {name: sum(g[0] * g[1] * b for g, b in launches(lines)) for name, (rc, lines) in seen.items()}
    for experts in (1, 64, 512):
        # 32 lanes a token, or 64
        assert threads["route %d" % experts] >= many * 32 and threads["gradient %d" % experts] >= many * 64
    assert threads["quantise"] >= many * 4
    tokens = 2 ** 30 - 1
    assert sum(g[0] for g, _ in launches(seen["layer"][1], "combine")) == tokens
    assert sum(g[0] * b for g, b in launches(seen["layer"][1], "route_kernel")) >= tokens * 32
