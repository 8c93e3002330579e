"""Layers with 4-bit floating point weights: what their calls refuse, on a context without a device; calls that have nothing to do."""
import ctypes as C

import pytest

from paper_2602_17698_amd import binding as sb

A = 1 << 20                     # an address that is aligned to everything and never read


@pytest.fixture()
def ctx():
    c = sb.Context(device=-1)
    yield c
    c.close()


def form(rows=64, cols=128, codes=A, scales=A, ld_codes=None, ld_scales=None):
    return sb.Mx(codes, scales, rows, cols, cols // 2 if ld_codes is None else ld_codes, sb.mx_scale_pitch(cols) if ld_scales is None else ld_scales)


def call(name, ctx, *args):
    return getattr(sb.load(), "sbits_" + name)(ctx.h, *[C.addressof(a) if isinstance(a, C.Structure) else a for a in args])


def test_pitches():
    assert [sb.mx_scale_pitch(c) for c in (32, 128, 160, 4096, 4128)] == [4, 4, 8, 128, 132]
    assert [sb.mx_out_pitch(r) for r in (1, 8, 9, 4096)] == [8, 8, 16, 4096]


BAD_FORMS = [(dict(codes=None), -1), (dict(codes=A + 8), -1), (dict(scales=A + 2), -1), (dict(scales=None), -1), (dict(cols=100), -2),
             (dict(cols=0), -2), (dict(cols=1 << 25), -2), (dict(ld_codes=48), -1), (dict(ld_codes=72), -1), (dict(ld_scales=2), -1),
             (dict(ld_scales=6), -1), (dict(rows=-1), -1), (dict(ld_codes=-64), -1)]


@pytest.mark.parametrize("change,status", BAD_FORMS)
def test_matrices_that_are_refused(ctx, change, status):
    m = form(**change)
    assert call("mx_quantize", ctx, A, 1, 128, m, None, 0) == status
    assert call("mx_gemm", ctx, m, A, 128, None, 4, 0, A, 0, 64, None, 0) == status
    assert call("mx_gemm", ctx, form(), None, 0, m, 4, 0, A, 0, 64, None, 0) == status


@pytest.mark.parametrize("x,kind,ld,values,ld_v,status", [
    (None, 1, 128, None, 0, -1), (A + 4, 1, 128, None, 0, -1), (A, 2, 128, None, 0, -1), (A, 1, 120, None, 0, -1), (A, 1, 132, None, 0, -1),
    (A, 0, 130, None, 0, -1), (A, 0, 132, A, 120, -1), (A, 0, 132, A + 8, 128, -1), (A, 0, 132, A, 132, -1), (A, 1, 136, A, 128, -7)])
def test_quantise_refuses(ctx, x, kind, ld, values, ld_v, status):
    assert call("mx_quantize", ctx, x, kind, ld, form(), values, ld_v) == status


def test_product_refuses(ctx):
    w = form()
    good = [w, A, 128, None, 4, 0, A, 0, 64, None, 0]
    assert call("mx_gemm", ctx, *good) == sb.ERR_HIP                            # no device, nothing else wrong
    for at, value, status in ((0, None, -1), (1, None, -1), (1, A + 2, -1), (2, 120, -1), (2, 129, -1), (3, w, -1), (4, -1, -1), (4, 1 << 31, -1),
                              (5, 2, -1), (6, None, -1), (6, A + 8, -1), (7, 2, -1), (8, 56, -1), (8, 68, -1), (0, form(rows=0), -2)):
        args = list(good)
        args[at] = value
        assert call("mx_gemm", ctx, *args) == status, (at, value)
    assert call("mx_gemm", ctx, form(rows=63), A, 128, None, 4, 1, A, 0, 64, None, 0) == sb.ERR_BAD_SHAPE          # halves
    assert call("mx_gemm", ctx, w, None, 0, form(rows=3), 4, 0, A, 0, 64, None, 0) == sb.ERR_BAD_SHAPE             # fewer rows than the batch
    assert call("mx_gemm", ctx, w, None, 0, form(rows=4, cols=160), 4, 0, A, 0, 64, None, 0) == sb.ERR_BAD_SHAPE


def router(**k):
    return sb.Router(**{**dict(experts=16, top_k=4), **k})


BAD_ROUTERS = [(dict(experts=0), -2), (dict(experts=513), -2), (dict(top_k=0), -2), (dict(top_k=17), -2), (dict(experts=64, top_k=33), -2),
               (dict(groups=3), -2), (dict(groups=0), -2), (dict(groups=4, top_groups=5), -2), (dict(groups=4, top_groups=0), -2),
               (dict(groups=8, top_groups=1), -2), (dict(experts=512, groups=128, top_groups=128), -2), (dict(scoring=2), -1), (dict(group_score=7), -1)]


@pytest.mark.parametrize("change,status", BAD_ROUTERS)
def test_routers_that_are_refused(ctx, change, status):
    r = router(**change)
    assert call("route", ctx, r, A, 0, 1024, None, 3, A, A) == status
    assert call("route_backward", ctx, r, A, 0, 1024, A, A, 3, A, 1024) == status
    assert call("expert_layer_ws_bytes", ctx, r, 3, form(16 * 64, 64), form(16 * 64, 32), 0) == 0


def test_routing_refuses(ctx):
    r = router()
    good = [r, A, 0, 16, None, 3, A, A]
    assert call("route", ctx, *good) == sb.ERR_HIP
    for at, value in ((0, None), (1, None), (1, A + 2), (2, 5), (3, 15), (4, A + 2), (5, -1), (5, 1 << 31), (6, None), (6, A + 1), (7, None)):
        args = list(good)
        args[at] = value
        assert call("route", ctx, *args) == sb.ERR_INVALID_ARG, (at, value)
    good = [r, A, 1, 16, A, A, 3, A, 16]
    assert call("route_backward", ctx, *good) == sb.ERR_HIP
    for at, value in ((1, None), (1, A + 1), (2, -1), (3, 15), (4, None), (5, None), (6, -1), (7, None), (7, A + 2), (8, 15)):
        args = list(good)
        args[at] = value
        assert call("route_backward", ctx, *args) == sb.ERR_INVALID_ARG, (at, value)


def test_layer_refuses(ctx):
    r, up, down = router(), form(16 * 2 * 32, 64), form(16 * 64, 32)
    need = call("expert_layer_ws_bytes", ctx, r, 5, up, down, 0)
    assert need > 0 and call("expert_layer_ws_bytes", ctx, r, 5, up, down, 1) > need
    good = [r, A, 0, 16, None, A, 64, 5, up, down, A, 64, A, A, 0, A, need]
    assert call("expert_layer", ctx, *good) == sb.ERR_HIP
    for at, value, status in ((0, None, -1), (1, None, -1), (2, 3, -1), (3, 8, -1), (4, A + 1, -1), (5, None, -1), (5, A + 8, -1), (6, 60, -1),
                              (7, -1, -1), (7, 1 << 29, -2), (7, 1 << 62, -1), (8, form(16 * 2 * 32, 96), -2), (8, form(16 * 2 * 32 - 1, 64), -2),
                              (9, form(16 * 64, 64), -2), (9, None, -1), (10, None, -1), (11, 60, -1), (12, None, -1), (13, A + 2, -1),
                              (14, 2, -1), (15, None, -5), (15, A + 128, -5), (16, need - 1, -5)):
        args = list(good)
        args[at] = value
        assert call("expert_layer", ctx, *args) == status, (at, value)


def test_calls_without_rows_do_nothing(ctx):
    r = router()
    assert call("mx_quantize", ctx, None, 1, 128, form(rows=0, codes=None, scales=None), None, 0) == sb.OK
    assert call("mx_gemm", ctx, form(), None, 0, None, 0, 0, None, 0, 64, None, 0) == sb.OK
    assert call("route", ctx, r, None, 0, 16, None, 0, None, None) == sb.OK
    assert call("route_backward", ctx, r, None, 0, 16, None, None, 0, None, 16) == sb.OK
    assert call("expert_layer", ctx, r, None, 0, 16, None, None, 64, 0, form(16 * 64, 64), form(16 * 64, 32), None, 64, None, None, 0, None, 0) == sb.OK
    assert call("mx_quantize", sb.Context(-1), A, 1, 128, None, None, 0) == sb.ERR_INVALID_ARG


def test_the_binding_checks_types_and_shapes(ctx):
    torch = pytest.importorskip("torch")
    u8 = lambda *s: torch.zeros(*s, dtype=torch.uint8)  # noqa: E731
    w = sb.mx(u8(64, 64), u8(64, 4), 128)
    x, y = torch.zeros(3, 128, dtype=torch.bfloat16), torch.zeros(3, 64)
    for wrong, error in ((lambda: ctx.mx_gemm(w, x.float(), y, None), TypeError), (lambda: ctx.mx_gemm(w, x, y.half(), None), TypeError),
                         (lambda: ctx.mx_gemm(w, x[:, :64], y, None), ValueError), (lambda: ctx.mx_gemm(w, x, y, None, gated=True), ValueError),
                         (lambda: ctx.mx_gemm(w, x.t().contiguous().t(), y, None), ValueError),
                         (lambda: ctx.mx_quantize(x, w), ValueError), (lambda: ctx.mx_quantize(x.half(), sb.mx(u8(3, 64), u8(3, 4), 128)), TypeError)):
        with pytest.raises(error):
            wrong()
    r, ids, weights, logits = router(), torch.zeros(3, 4, dtype=torch.int32), torch.zeros(3, 4), torch.zeros(3, 16)
    for args, error in (((logits, None, ids.long(), weights), TypeError), ((logits, None, ids, weights.double()), TypeError),
                        ((logits[:, :15], None, ids, weights), ValueError), ((logits, torch.zeros(15), ids, weights), ValueError),
                        ((logits, None, ids[:, :3], weights[:, :3]), ValueError), ((logits[:2], None, ids, weights), ValueError),
                        ((logits.half(), None, ids, weights), TypeError), ((logits, None, ids.t().contiguous().t(), weights), ValueError)):
        with pytest.raises(error):
            ctx.route(r, *args)
