"""Descriptors of matrices in the microscaled form: what tensors they are made of."""
import pytest

from paper_2602_17698_amd import binding as sb

torch = pytest.importorskip("torch")


def u8(*shape):
    return torch.zeros(*shape, dtype=torch.uint8)


def test_descriptors_of_dense_and_of_wider_tensors():
    for codes, scales, cols in ((u8(3, 80), u8(3, 8), 160), (u8(3, 96)[:, :80], u8(3, 16)[:, :8], 160), (u8(0, 16), u8(0, 4), 32)):
        d = sb.mx(codes, scales, cols)
        assert (d.codes or 0, d.scales or 0) == (codes.data_ptr(), scales.data_ptr())
        assert (d.rows, d.cols, d.ld_codes, d.ld_scales) == (codes.shape[0], cols, codes.stride(0), scales.stride(0))


@pytest.mark.parametrize("kind", [torch.int8, torch.int32, torch.float32, torch.bfloat16])
def test_other_types_are_refused(kind):
    with pytest.raises(TypeError):
        sb.mx(u8(3, 80).to(kind), u8(3, 8), 160)
    with pytest.raises(TypeError):
        sb.mx(u8(3, 80), u8(3, 8).to(kind), 160)


@pytest.mark.parametrize("codes,scales,cols", [((3, 80), (2, 8), 160), ((3, 80), (4, 8), 160), ((3, 64), (3, 8), 160), ((3, 80), (3, 4), 160), ((3, 80), (3, 5), 160),
                                               ((3, 0), (3, 0), 32)])
def test_tensors_that_do_not_hold_the_matrix_are_refused(codes, scales, cols):
    with pytest.raises(ValueError):
        sb.mx(u8(*codes), u8(*scales), cols)
    # (pitches that are long enough do not help: the last row ends with its tensor)
    with pytest.raises(ValueError):
        sb.mx(u8(codes[0], 256)[:, :codes[1]], u8(scales[0], 64)[:, :scales[1]], cols)


def test_rows_that_are_not_dense_are_refused():
    with pytest.raises(ValueError):
        sb.mx(u8(80, 3).t(), u8(3, 8), 160)
    with pytest.raises(ValueError):
        sb.mx(u8(3, 80), u8(3, 16)[:, ::2], 160)
