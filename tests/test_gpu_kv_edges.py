"""Attention to the microscaled cache where its masks, tables and values are at their borders, against 64 bits."""
import math

import pytest
import torch

import kv_tight
from kv_plain import Batch
from paper_2602_17698_amd import binding as sb

pytestmark = pytest.mark.gpu
BF16 = torch.bfloat16


@pytest.fixture(scope="module")
def ctx():
    c = sb.Context(0, torch.cuda.current_stream().cuda_stream)
    yield c
    c.close()


def queries(b, heads, seed=1):
    return (torch.randn(b.tokens, heads, b.dim, generator=torch.Generator().manual_seed(seed)) * 1.5).to(BF16)


def attend(ctx, b, q, lse=True, hints=(), **k):
    """out and lse on the CPU; where nothing is written 77."""
    cache, seqs, _ = b.on(sb, **dict(hints))
    out = torch.full(q.shape, 77.0, dtype=BF16, device="cuda")
    sums = torch.full(q.shape[:2], 77.0, device="cuda") if lse else None
    ws = torch.full((max(1, ctx.kv_attention_ws_bytes(cache, seqs, b.tokens, q.shape[1])),), 255, dtype=torch.uint8, device="cuda")
    ctx.kv_attention(cache, seqs, q.cuda(), out, ws, lse=sums, **k)
    return out.cpu(), sums.cpu() if lse else None


def check(ctx, b, q, hints=(), lse=True, **k):
    out, sums = attend(ctx, b, q, lse, hints, **k)
    want, want_lse, off, off_lse = kv_tight.attention(b, q, terms=4 if lse else 3, **k)
    rows = b.rows()
    got, nan = out[rows].double(), torch.isnan(want)
    assert torch.equal(torch.isnan(got), nan)
    assert ((got - want).abs() <= off)[~nan].all(), float(((got - want).abs() / off.clamp(min=1e-30))[~nan].max())
    if lse:
        none = want_lse == -math.inf
        assert (sums[rows][none] == -math.inf).all()
        assert ((sums[rows] - want_lse).abs() <= off_lse)[~none & ~torch.isnan(want_lse)].all()
    return out, sums


# ---- a table that ends ahead of the sequence -------------------------------------------------------
@pytest.mark.parametrize("window", [0, 1, 20, 64, 150])
@pytest.mark.parametrize("sizes", [[(1, 999), (2, 60)], [(70, 900), (3, 10)], [(150, 0)]])
@pytest.mark.parametrize("pages", [1, 5])
def test_a_window_behind_the_end_of_the_table(ctx, window, sizes, pages):
    """The last rows' windows begin behind the last page that the table has: nothing is there for them."""
    b = Batch(sizes, 16, 2, 64, seed=window + pages, lead=1, behind=1)
    b.table = b.table[:, :pages].contiguous()
    out, sums = check(ctx, b, queries(b, 4), window=window)
    if window and sizes[0][1] == 900 or sizes[0][0] == 1 and window:
        assert (out[1] == 0).all() and (sums[1] == -math.inf).all()
    check(ctx, b, queries(b, 4), window=window, lse=False, hints=dict(max_new=max(n for n, _ in sizes)))
