"""Tensors of one row, whatever their distance to a next one."""
import pytest

from paper_2602_17698_amd import binding as sb

torch = pytest.importorskip("torch")


@pytest.fixture()
def ctx():
    c = sb.Context(device=-1)               # no device: what passes all checks ends with ERR_HIP
    yield c
    c.close()


def no_device(call):
    with pytest.raises(sb.SbitsError) as e:
        call()
    assert e.value.status == sb.ERR_HIP


def one_row(cols, kind):
    """[1, cols], as the transpose of a column: its rows are one element apart."""
    t = torch.zeros(cols, 1, dtype=kind).t()
    assert t.shape == (1, cols) and t.stride() == (1, 1)
    return t


def test_one_row_needs_no_pitch(ctx):
    bf16, u8, f32 = torch.bfloat16, torch.uint8, torch.float32
    w = sb.mx(torch.zeros(40, 80, dtype=u8), torch.zeros(40, 8, dtype=u8), 160)
    no_device(lambda: ctx.mx_gemm(w, one_row(160, bf16), one_row(40, f32), None))
    q = sb.mx(one_row(80, u8), one_row(8, u8), 160)
    no_device(lambda: ctx.mx_quantize(one_row(160, bf16), q, one_row(160, bf16)))
    no_device(lambda: ctx.mx_gemm(w, q, one_row(40, bf16), None))
    r = sb.Router(experts=9, top_k=2)
    ids, weights = torch.zeros(1, 2, dtype=torch.int32), torch.zeros(1, 2)
    no_device(lambda: ctx.route(r, one_row(9, f32), None, ids, weights))
    no_device(lambda: ctx.route_backward(r, one_row(9, bf16), ids, weights, one_row(9, f32)))


def test_rows_a_short_way_apart_are_still_refused(ctx):
    r = sb.Router(experts=9, top_k=2)
    ids, weights = torch.zeros(2, 2, dtype=torch.int32), torch.zeros(2, 2)
    with pytest.raises(sb.SbitsError) as e:
        ctx.route(r, torch.zeros(10).as_strided((2, 9), (1, 1)), None, ids, weights)
    assert e.value.status == sb.ERR_INVALID_ARG
