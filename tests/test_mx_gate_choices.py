"""Which kernels the tests of the gate run: few rows, tiles of 64, 128 and 256, parts of the columns."""
from recording_runtime import record
from test_gpu_mx_gate import SHAPES
from test_mx_choices import tile_rows

GATED = r"""
import ctypes as C
out = []
ctx = sb.Context(0, 0)
for batch, outs, cols in %r:
    for four in (0, 1):
        pitch = sb.mx_scale_pitch(cols)
        w = sb.Mx(fake(2 * outs * cols), fake(2 * outs * pitch), 2 * outs, cols, cols // 2, pitch)
        x = sb.Mx(fake(batch * cols), fake(batch * pitch), batch, cols, cols // 2, pitch)
        need = ctx.mx_gemm_ws_bytes(w, batch, bool(four), True)
        log()
        rc = sb.load().sbits_mx_gemm(ctx.h, C.addressof(w), None if four else fake(batch * cols * 2), cols, C.addressof(x) if four else None,
                                     batch, 1, fake(batch * outs * 4), 0, sb.mx_out_pitch(outs), fake(need + 256), need)
        out.append([batch, outs, cols, rc, [line.split()[1] for line in log() if line.startswith("launch")]])
answer(out)
"""


def test_gated_products_run_the_kernels_that_their_tests_are_for(tmp_path):
    want = dict(zip(SHAPES, ((16, 1), (16, 1), (64, 1), (128, 1), (256, 1), (64, 2))))
    for *shape, rc, names in record(tmp_path, GATED % (SHAPES,)):
        assert rc == 0 and (tile_rows(names[0]), len(names)) == want[tuple(shape)], (shape, names)
        assert ("mx_join" in names[-1]) == (len(names) == 2)
