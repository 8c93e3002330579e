"""Products of 4-bit activations with powers of two from one end of the bytes to the other, and matrices with blocks that were not finite when they were quantised."""
import math

import pytest
import torch

import mx_plain as mp
from paper_2602_17698_amd import binding as sb

pytestmark = pytest.mark.gpu
BYTES = [0, 1, 2, 40, 100, 126, 127, 128, 160, 220, 253, 254]


@pytest.fixture(scope="module")
def ctx():
    c = sb.Context(0, torch.cuda.current_stream().cuda_stream)
    yield c
    c.close()


@pytest.mark.parametrize("batch,rows,cols", [(12, 12, 64), (12, 60, 4096), (1020, 1032, 288)])
@pytest.mark.parametrize("gated", [False, True])
def test_powers_of_both_operands(ctx, batch, rows, cols, gated):
    """A power for each row: sums from far below fp32's least number to beyond its largest."""
    g = torch.Generator().manual_seed(rows)
    code, xc = (torch.randint(0, 16, (n, cols), generator=g).to(torch.uint8) for n in (2 * rows if gated else rows, batch))
    powers = torch.tensor(BYTES, dtype=torch.uint8)
    byte = powers[torch.arange(code.shape[0]) % 12][:, None].repeat(1, cols // 32)
    xb = powers[torch.arange(batch) * 5 % 12][:, None].repeat(1, cols // 32)
    w, x = (sb.mx(*mp.stored(c, b, "cuda")) for c, b in ((code, byte), (xc, xb)))
    y = torch.empty(batch, sb.mx_out_pitch(rows), device="cuda")
    ws = torch.empty(max(256, ctx.mx_gemm_ws_bytes(w, batch, True, gated)), dtype=torch.uint8, device="cuda")
    print("[case]", batch, rows, cols, gated, flush=True)
    ctx.mx_gemm(w, x, y[:, :rows], ws, gated=gated)
    w64, x64 = mp.values(code, byte), mp.values(xc, xb)
    want, off = mp.product(x64, w64, gated)
    # sums whose terms are all within fp32, and its gate's products; below the least normal number a term, a sum or silu may be 0
    small = (x64.abs() @ w64.abs().T) < 2.0 ** 127
    if gated:
        a, b = small.chunk(2, 1)
        small = a & b & (want.abs() < 2.0 ** 127)
        u = (x64 @ w64.T).chunk(2, 1)[1]
        off = off + 2.0 ** -126 * (1 + cols) * (1 + u.abs())
    off = off + 2.0 ** -126 * (1 + cols)
    got = y[:, :rows].cpu().double()
    assert bool(small.any()) and bool(torch.isfinite(got[small]).all())
    assert bool(((got - want).abs() <= off + 2.0 ** -24 * (want.abs() + off))[small].all())


@pytest.mark.parametrize("batch,rows,cols", [(1, 40, 96), (700, 2050, 416), (4000, 1030, 416), (60, 250, 14336)])
@pytest.mark.parametrize("four", [False, True])
def test_matrices_with_blocks_that_were_not_finite(ctx, batch, rows, cols, four):
    """Quantised from a NaN or an infinity: codes 0 and the byte 255, and all of their row's outputs NaN."""
    g = torch.Generator().manual_seed(rows)
    w = torch.randn(rows, cols, generator=g)
    w[3, cols - 1], w[17, 0], w[rows - 1, 40] = math.nan, math.inf, -math.inf
    x = torch.randn(batch, cols, generator=g).to(torch.bfloat16)
    q = sb.mx(torch.empty(rows, cols // 2, dtype=torch.uint8, device="cuda"), torch.empty(rows, sb.mx_scale_pitch(cols), dtype=torch.uint8, device="cuda"), cols)
    ctx.mx_quantize(w.cuda(), q)
    xd = sb.mx(*mp.stored(*mp.quantise(x), "cuda")) if four else x.cuda()
    y = torch.empty(batch, sb.mx_out_pitch(rows), device="cuda")
    ctx.mx_gemm(q, xd, y[:, :rows], torch.empty(max(256, ctx.mx_gemm_ws_bytes(q, batch, four)), dtype=torch.uint8, device="cuda"))
    broken = torch.zeros(rows, dtype=torch.bool)
    broken[3] = broken[17] = broken[rows - 1] = True
    got = y[:, :rows].cpu()
    assert bool(torch.isnan(got[:, broken]).all()) and bool(torch.isfinite(got[:, ~broken]).all())
