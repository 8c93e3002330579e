"""Which kernels the products and layers of the GPU tests run: chosen by estimates on the host, seen here without a device."""
import re

from mx_shapes import LARGE, LARGE_LAYERS, LAYERS, SHAPES
from recording_runtime import record

PRODUCTS = r"""
import ctypes as C
out = []
ctx = sb.Context(0, 0)
for batch, rows, cols in %r:
    for four in (0, 1):
        pitch = sb.mx_scale_pitch(cols)
        w = sb.Mx(fake(rows * cols), fake(rows * pitch), rows, cols, cols // 2, pitch)
        x = sb.Mx(fake(batch * cols), fake(batch * pitch), batch, cols, cols // 2, pitch)
        need = ctx.mx_gemm_ws_bytes(w, batch, bool(four))
        log()
        call = lambda given: sb.load().sbits_mx_gemm(ctx.h, C.addressof(w), None if four else fake(batch * cols * 2), cols, C.addressof(x) if four else None,
                                                     batch, 0, fake(batch * rows * 4), 0, sb.mx_out_pitch(rows), fake(need + 256), given)
        rc = call(need)
        launches = [line.split() for line in log() if line.startswith("launch")]
        short = call(need - 1) if need else -5
        out.append([batch, rows, cols, four, rc, short, need, [[k[1], k[3]] for k in launches], len(log()) if need else 0])
answer(out)
"""


def tile_rows(name):
    many = re.search(r"mx_gemm_many_kernelILb\dELb\dELi(\d)E", name)
    return 64 * int(many.group(1)) if many else 16


def test_products_run_the_kernels_that_their_tests_are_for(tmp_path):
    large = {k[:3]: k[3:] for k in LARGE}
    seen = set()
    for batch, rows, cols, four, rc, short, need, launches, after in record(tmp_path, PRODUCTS % (SHAPES + list(large),)):
        assert rc == 0 and short == -5 and after == 0
        names = [k[0] for k in launches]
        tile, parts = large.get((batch, rows, cols), (16, (False, False)))
        assert tile_rows(names[0]) == tile, (batch, rows, cols, four)
        assert (need > 0) == parts[four] == any("mx_join" in n for n in names) and len(names) == 1 + parts[four], (batch, rows, cols, four)
        seen.add(names[0].split("kernel")[1])
    # few rows: x in bf16 and 4 bits, by 4 and 8 waves, 1, 2 and 4 tiles of W
    for x4 in (0, 1):
        for waves in ("4", "8"):
            for tiles in "124":
                assert any(n.startswith("ILb%dELb0ELi%sELi%sE" % (x4, waves, tiles)) for n in seen), (x4, waves, tiles)


LAYER = r"""
import ctypes as C
out = []
ctx = sb.Context(0, 0)
for tokens, experts, top_k, hidden, inner in %r:
    for four in (0, 1):
        r = sb.Router(experts, top_k)
        up = sb.Mx(fake(experts * inner * hidden), fake(experts * inner * hidden), experts * 2 * inner, hidden, hidden // 2, sb.mx_scale_pitch(hidden))
        down = sb.Mx(fake(experts * inner * hidden), fake(experts * inner * hidden), experts * hidden, inner, inner // 2, sb.mx_scale_pitch(inner))
        need = ctx.expert_layer_ws_bytes(r, tokens, up, down, bool(four))
        log()
        rc = sb.load().sbits_expert_layer(ctx.h, C.addressof(r), fake(tokens * experts * 4), 0, experts, None, fake(tokens * hidden * 2), hidden, tokens,
                                          C.addressof(up), C.addressof(down), fake(tokens * hidden * 2), hidden, fake(tokens * top_k * 4),
                                          fake(tokens * top_k * 4), four, fake(need), need)
        out.append([tokens, experts, top_k, hidden, inner, rc, [line.split()[1] for line in log() if line.startswith("launch")]])
answer(out)
"""


def test_layers_run_the_kernels_that_their_tests_are_for(tmp_path):
    large = {k[:5]: k[5] for k in LARGE_LAYERS}
    for *shape, rc, names in record(tmp_path, LAYER % (LAYERS + list(large),)):
        products = [n for n in names if "gemm" in n]
        assert rc == 0 and len(products) == 2
        assert [tile_rows(n) for n in products] == [large.get(tuple(shape), 16)] * 2, shape
