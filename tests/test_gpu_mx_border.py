"""Matrices that end just within, and just beyond, what the product of many rows addresses: the last rows are read like the first."""
import pytest
import torch

import mx_plain as mp
from paper_2602_17698_amd import binding as sb

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("rows", [299592, 299593])
@pytest.mark.parametrize("four", [False, True])
def test_last_rows_of_a_matrix_of_2_gib(rows, four):
    ctx = sb.Context(0, torch.cuda.current_stream().cuda_stream)
    cols, batch, some = 14336, 130, 96
    g = torch.Generator(device="cuda").manual_seed(rows)
    codes = torch.randint(0, 256, (rows, cols // 2), dtype=torch.uint8, device="cuda", generator=g)
    scales = torch.randint(117, 124, (rows, sb.mx_scale_pitch(cols)), dtype=torch.uint8, device="cuda", generator=g)
    x = torch.randn(batch, cols, device="cuda", generator=g).to(torch.bfloat16)
    w = sb.mx(codes, scales, cols)
    if four:
        xc, xb = mp.quantise(x.cpu())
        xs, xd = mp.values(xc, xb), sb.mx(*mp.stored(xc, xb, "cuda"))
    else:
        xs, xd = x.cpu().double(), x
    y = torch.empty(batch, sb.mx_out_pitch(rows), device="cuda")[:, :rows]
    print("[case]", rows, four, flush=True)
    ctx.mx_gemm(w, xd, y, torch.empty(max(256, ctx.mx_gemm_ws_bytes(w, batch, four)), dtype=torch.uint8, device="cuda"))
    for part in (slice(0, some), slice(rows - some, rows)):
        want, off = mp.product(xs, mp.values(mp.unpack(codes[part].cpu()), scales[part, :cols // 32].cpu()), False)
        assert bool(((y[:, part].cpu().double() - want).abs() <= off).all())
    ctx.close()
