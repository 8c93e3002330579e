"""Rotations of few heads and many tokens, several rows to a workgroup: against 64 bits, and bit by bit against a row a workgroup."""
import pytest
import torch

import kv_plain
from paper_2602_17698_amd import binding as sb

pytestmark = pytest.mark.gpu
BF16, FP32 = torch.bfloat16, torch.float32


@pytest.mark.parametrize("dtype", [BF16, FP32])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("tokens,heads,dim,dims,pad,back", [
    (100003, 1, 64, 64, 0, False), (60001, 2, 64, 64, 8, True), (70000, 1, 32, 32, 0, True), (50001, 1, 256, 256, 0, False), (40001, 3, 80, 38, 0, False),
    (30011, 1, 7, 6, 3, True), (1025, 1, 64, 16, 1, False), (200003, 1, 2, 2, 0, False), (2047, 5, 96, 96, 0, True), (50000, 7, 128, 128, 16, False),
    (33333, 1, 96, 16, 0, False)])
def test_few_heads(dtype, interleaved, tokens, heads, dim, dims, pad, back):
    ctx = sb.Context(0, torch.cuda.current_stream().cuda_stream)
    g = torch.Generator().manual_seed(tokens)
    x = torch.randn(tokens, heads, dim, generator=g).to(dtype)
    at = torch.randint(-1000, 1 << 20, (tokens,), generator=g).int()
    turns = kv_plain.turns(dims)
    r = sb.rotary(torch.tensor(turns, dtype=torch.float64, device="cuda"), interleaved, 1.25)
    base = torch.full((tokens, heads * dim + pad), 77.0, dtype=dtype, device="cuda")
    out = base[:, :heads * dim].unflatten(1, (heads, dim))
    src, positions = x.cuda(), at.cuda()
    ctx.rotate(r, positions, src, out, inverse=back)
    assert (base[:, heads * dim:] == 77).all()
    rows = torch.cat([torch.arange(40), torch.randint(0, tokens, (100,), generator=g), torch.arange(tokens - 40, tokens)])
    want, size = kv_plain.turn(x[rows], at[rows], turns, interleaved, 1.25, back)
    # as for any rotation: cos and sin, a product and the sum round, and the output
    off = 4 * 2.0 ** -24 * size + (2.0 ** -8 * want.abs() if dtype == BF16 else 0.0)
    off[..., dims:] = 0
    assert ((out.cpu()[rows].double() - want).abs() <= off).all()
    other = torch.empty_like(src)
    for i in range(0, tokens, 800):                              # (calls of so few rows take one to a workgroup)
        ctx.rotate(r, positions[i:i + 800], src[i:i + 800], other[i:i + 800], inverse=back)
    assert torch.equal(out, other)
    ctx.rotate(r, positions, src, src, inverse=back)             # in place
    assert torch.equal(src, other)
    ctx.close()
