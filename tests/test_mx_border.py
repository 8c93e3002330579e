"""Products of many rows address a matrix by 31 bits, from a little ahead of its begin: which sizes they are given, on both sides of the border."""
from recording_runtime import record
from test_mx_choices import tile_rows

PRODUCTS = r"""
import ctypes as C
out = []
ctx = sb.Context(0, 0)
for rows, cols, batch in %r:
    pitch = sb.mx_scale_pitch(cols)
    for four in (0, 1):
        w = sb.Mx(fake(rows * cols // 2), fake(rows * pitch), rows, cols, cols // 2, pitch)
        x = sb.Mx(fake(batch * cols), fake(batch * pitch), batch, cols, cols // 2, pitch)
        need = ctx.mx_gemm_ws_bytes(w, batch, bool(four))
        log()
        rc = sb.load().sbits_mx_gemm(ctx.h, C.addressof(w), None if four else fake(batch * cols * 2), cols, C.addressof(x) if four else None,
                                     batch, 0, fake(batch * rows * 4), 0, sb.mx_out_pitch(rows), fake(need + 256), need)
        out.append([rows, cols, four, rc, [line.split()[1] for line in log() if line.startswith("launch")]])
answer(out)
"""

# (rows of the last matrix below the border, columns, rows of x): codes end 3 KiB ahead of 2 GiB, or up to a row further ahead
BORDER = [(299592, 14336, 700), (1048574, 4096, 4000), (16777191, 256, 70)]


def test_matrices_at_the_border_of_31_bits(tmp_path):
    lead = 3 * 1024                                             # bytes that the kernel's buffers begin ahead
    cases = [(rows + more, cols, batch) for rows, cols, batch in BORDER for more in (0, 1)]
    for rows, cols, four, rc, names in record(tmp_path, PRODUCTS % (cases,)):
        inside = rows * (cols // 2) + lead <= 2 ** 31 - 1
        assert rc == 0 and inside == ((rows, cols) in [k[:2] for k in BORDER])
        assert (tile_rows(names[0]) > 16) == inside, (rows, cols, four, names)


LAYER = r"""
import ctypes as C
out = []
ctx = sb.Context(0, 0)
experts, top_k, hidden, inner = 4, 2, 1024, 64
up = sb.Mx(fake(1 << 20), fake(1 << 20), experts * 2 * inner, hidden, hidden // 2, sb.mx_scale_pitch(hidden))
down = sb.Mx(fake(1 << 20), fake(1 << 20), experts * hidden, inner, inner // 2, sb.mx_scale_pitch(inner))
r = sb.Router(experts, top_k)
for tokens in (1048574, 1048575):
    need = ctx.expert_layer_ws_bytes(r, tokens, up, down)
    log()
    rc = sb.load().sbits_expert_layer(ctx.h, C.addressof(r), fake(tokens * experts * 4), 0, experts, None, fake(tokens * hidden * 2), hidden, tokens,
                                      C.addressof(up), C.addressof(down), fake(tokens * hidden * 2), hidden, fake(tokens * top_k * 4),
                                      fake(tokens * top_k * 4), 0, fake(need), need)
    out.append([tokens, rc, [line.split()[1] for line in log() if line.startswith("launch") and "gemm" in line]])
answer(out)
"""


def test_tokens_at_the_border_of_31_bits(tmp_path):
    """A layer's gated product reads the tokens by a list, from the first of all."""
    near, far = record(tmp_path, LAYER)
    assert near[1] == 0 and all(tile_rows(n) > 16 for n in near[2])
    assert far[1] == 0 and all(tile_rows(n) == 16 for n in far[2])
