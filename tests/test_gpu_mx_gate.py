"""Gated products where the gate is far from 0: silu's ends, sums that are infinite, broken blocks; by the kernels of few and of many rows and of parts."""
import math

import pytest
import torch

import mx_plain as mp
from paper_2602_17698_amd import binding as sb

pytestmark = pytest.mark.gpu

# (batch, outputs, cols): few rows by 1 and by several tiles, many rows by tiles of 64, 128 and 256, parts of the columns
SHAPES = [(1, 40, 64), (16, 300, 96), (700, 1025, 800), (4000, 515, 288), (2000, 2050, 288), (60, 125, 14336)]


@pytest.fixture(scope="module")
def ctx():
    c = sb.Context(0, torch.cuda.current_stream().cuda_stream)
    yield c
    c.close()


def workspace(ctx, w, batch, four):
    return torch.full((max(256, ctx.mx_gemm_ws_bytes(w, batch, four, True)),), 0xff, dtype=torch.uint8, device="cuda")


@pytest.mark.parametrize("batch,outs,cols", SHAPES)
@pytest.mark.parametrize("four", [False, True])
@pytest.mark.parametrize("out", [torch.float32, torch.bfloat16])
def test_gate_at_its_ends(ctx, batch, outs, cols, four, out):
    """Three terms that are not zero make an output: g = wg (x0 + x1), u = wu x32, exact in fp32 or infinite.  Among the g: up to 3e38 either way, where e^-g is
    0 or infinite; -87.4 .. -88.7, where 1 + e^-g is above 2^126; sums beyond fp32."""
    g = torch.Generator().manual_seed(batch + cols)
    gs = [(0.0, 0.0), (1.0, 0.0), (-1.5, 0.0), (16.0, 4.0), (-16.0, -4.0), (64.0, 16.0), (-64.0, -16.0), (-64.0, -24.0), (-48.0, -48.0), (-128.0, 0.0), (-1024.0, 0.0),
          (1024.0, 0.0), (1.5 * 2.0 ** 126, 0.0), (1.5 * 2.0 ** 127, 0.0), (-1.5 * 2.0 ** 127, 0.0), (1.5 * 2.0 ** 127, -0.0)]
    if not four:
        gs += [(2.3e38, 0.0), (2.4e38, 0.0), (3e38, 0.0), (-3e38, 0.0), (-87.5, 0.0), (-88.5, 0.0), (-84.0, 0.0)]
    us = [1.0, -2.0, 1.5 * 2.0 ** -100, -3.0 * 2.0 ** -126, 2.0 ** 90, 0.0]
    some = torch.randint(0, len(gs), (batch,), generator=g)
    some[:min(batch, len(gs))] = torch.arange(min(batch, len(gs))) if batch > 1 else len(gs) - 1
    x = torch.zeros(batch, cols, dtype=torch.float64)
    x[:, :2] = torch.tensor(gs, dtype=torch.float64)[some]
    x[:, 32] = torch.tensor(us, dtype=torch.float64)[torch.randint(0, len(us), (batch,), generator=g)]
    x = x.to(torch.bfloat16)
    if batch == 1:
        x[0, 0], x[0, 1], x[0, 32] = 1.5 * 2.0 ** 127, 0.0, 1.5 * 2.0 ** -100
    code = torch.zeros(2 * outs, cols, dtype=torch.uint8)
    code[:outs, 0] = torch.randint(2, 8, (outs,), generator=g).to(torch.uint8)
    code[0, 0] = code[outs - 1, 0] = 2
    code[:outs, 1] = code[:outs, 0]
    code[outs:, 32] = torch.randint(2, 16, (outs,), generator=g).to(torch.uint8)
    byte = torch.full((2 * outs, cols // 32), 127, dtype=torch.uint8)
    w = sb.mx(*mp.stored(code, byte, "cuda"))
    if four:
        xc, xb = mp.quantise(x)
        assert torch.equal(mp.values(xc, xb), x.double())                   # every value has a code
        xd = sb.mx(*mp.stored(xc, xb, "cuda"))
    else:
        xd = x.cuda()
    y = torch.empty(batch, sb.mx_out_pitch(outs), dtype=out, device="cuda")
    print("[case]", batch, outs, cols, four, out, flush=True)
    ctx.mx_gemm(w, xd, y[:, :outs], workspace(ctx, w, batch, four), gated=True)
    got = y[:, :outs].cpu().double()
    weights = mp.values(code, byte)
    x64 = x.double()
    gate = (x64[:, :1] * weights[:outs, 0] + x64[:, 1:2] * weights[:outs, 1]).float().double()        # (infinite beyond fp32)
    u = x64[:, 32:33] * weights[outs:, 32]
    silu = gate / (1 + torch.exp(-gate))
    want = silu * u
    # the hardware's exp and reciprocal are off by a unit in the last place each, which is two roundings; besides a sum, a correction and two products: 8.
    # silu below the least normal number may be 0
    off = 8 * 2.0 ** -24 * want.abs() + 2.0 ** -126 * u.abs() + 2.0 ** -149
    if out == torch.bfloat16:
        off = off + (2.0 ** -8 * (want.abs() + off)).clamp(min=2.0 ** -134)       # (half a step, of numbers below 2^-126, too)
    border = (want.abs() * 2.0 ** -128 - 1).abs() < 2.0 ** -20            # as large as the first number beyond fp32: that, or infinite
    assert bool((got.abs() > 3.38e38)[border].all()) and torch.equal(got.sign()[border], want.sign()[border])
    got = torch.where(border, want, got)
    want = torch.where((want.abs() > 2.0 ** 128) & ~border, want * math.inf, want)
    fine = torch.isfinite(want)
    assert bool(((got - want).abs() <= off)[fine].all()), float(((got - want).abs() / off)[fine].max())
    assert torch.equal(torch.nan_to_num(got[~fine], nan=5.0, posinf=7.0, neginf=-7.0), torch.nan_to_num(want[~fine], nan=5.0, posinf=7.0, neginf=-7.0))
    assert bool((fine & (gate > 2.36e38)).any()) or batch == 16


@pytest.mark.parametrize("batch,outs,cols", [(2, 150, 416), (700, 1025, 416), (4000, 515, 416), (2000, 2050, 416), (60, 150, 14336)])
@pytest.mark.parametrize("four", [False, True])
def test_broken_blocks_of_gated_products(ctx, batch, outs, cols, four):
    """A block with the byte 255 in either half of W makes its output NaN for all rows of x, a broken block of x its row; the others are as without."""
    g = torch.Generator().manual_seed(6)
    code, byte = mp.random_matrix(2 * outs, cols, g)
    x = torch.randn(batch, cols, generator=g).to(torch.bfloat16)

    def run(byte, x):
        w = sb.mx(*mp.stored(code, byte, "cuda"))
        xd = sb.mx(*mp.stored(*mp.quantise(x), "cuda")) if four else x.cuda()
        y = torch.empty(batch, sb.mx_out_pitch(outs), device="cuda")
        ctx.mx_gemm(w, xd, y[:, :outs], workspace(ctx, w, batch, four), gated=True)
        return y[:, :outs].cpu()
    good = run(byte, x)
    byte2, x2 = byte.clone(), x.clone()
    byte2[17, 12], byte2[outs + 99, 0], x2[1, 415] = 255, 255, math.nan
    bad = run(byte2, x2)
    hit = torch.zeros(batch, outs, dtype=torch.bool)
    hit[:, 17] = hit[:, 99] = True
    hit[1] = True
    assert bool(torch.isfinite(good).all()) and bool(torch.isnan(bad[hit]).all())
    assert torch.equal(bad[~hit], good[~hit])
