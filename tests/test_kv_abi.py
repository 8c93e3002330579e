"""The cache of keys and values, rotary positions and attention: what their calls refuse, on a context without a device; calls that have nothing to do."""
import ctypes as C
import math

import pytest
import torch

import kv_plain
from paper_2602_17698_amd import binding as sb

A = 1 << 20                     # an address that is aligned to everything and never read


@pytest.fixture()
def ctx():
    c = sb.Context(device=-1)
    yield c
    c.close()


def cache(pages=8, page_tokens=16, kv_heads=2, head_dim=128, **k):
    rows = kv_heads * page_tokens
    d = dict(k_codes=A, k_scales=A, v_codes=A, v_scales=A, pages=pages, ld_codes=rows * head_dim // 2, ld_scales=rows * sb.mx_scale_pitch(max(head_dim, 1)),
             page_tokens=page_tokens, kv_heads=kv_heads, head_dim=head_dim)
    d.update(k)
    return sb.KvCache(*[d[f] for f, _ in sb.KvCache._fields_])


def seqs(**k):
    d = dict(starts=A, lengths=A, pages=A, ld_pages=4, count=3, max_pages=4, max_new=0, max_length=0)
    d.update(k)
    return sb.Sequences(*[d[f] for f, _ in sb.Sequences._fields_])


def turns(**k):
    d = dict(turns=A, pairs=64, interleaved=0, amplitude=1.0)
    d.update(k)
    return sb.Rotary(*[d[f] for f, _ in sb.Rotary._fields_])


def call(name, ctx, *args):
    return getattr(sb.load(), "sbits_" + name)(ctx.h if ctx else None, *[C.addressof(a) if isinstance(a, C.Structure) else a for a in args])


def store(ctx, c=None, s=None, change=(), rotary=None, positions=None, q=None, q_heads=0, q_out=None):
    args = [c or cache(), s or seqs(), 5, A, 256, 128, A, 256, 128, 1, rotary, positions, q, 512, 128, q_heads, q_out, 512, 128]
    for at, value in change:
        args[at] = value
    return call("kv_store", ctx, *args)


def attend(ctx, c=None, s=None, change=()):
    args = [c or cache(), s or seqs(), 5, 8, A, 1024, 128, 0.1, 1, 0, A, 1024, 128, None, A, 1 << 40]
    for at, value in change:
        args[at] = value
    return call("kv_attention", ctx, *args)


def load(ctx, c=None, s=None, change=()):
    args = [c or cache(), s or seqs(), 5, A, 256, 128, A, 256, 128, 1]
    for at, value in change:
        args[at] = value
    return call("kv_load", ctx, *args)


def everything(ctx, c=None, s=None):
    return {store(ctx, c, s), attend(ctx, c, s), load(ctx, c, s)}


def test_nothing_wrong_but_no_device(ctx):
    assert everything(ctx) == {sb.ERR_HIP}
    assert everything(ctx, cache(page_tokens=8, kv_heads=1, head_dim=32)) != {0}
    assert store(ctx, rotary=turns(), positions=A, q=A, q_heads=8, q_out=A) == sb.ERR_HIP
    assert call("rotate", ctx, turns(), A, 3, 2, 128, A, 256, 128, 1, 0, A, 256, 128) == sb.ERR_HIP


@pytest.mark.parametrize("change,status", [
    (dict(k_codes=None), -1), (dict(v_codes=A + 8), -1), (dict(k_scales=A + 2), -1), (dict(v_scales=None), -1), (dict(pages=0), -2), (dict(pages=1 << 31), -2),
    (dict(page_tokens=4), -2), (dict(page_tokens=24), -2), (dict(page_tokens=1 << 21), -2), (dict(kv_heads=0), -2), (dict(kv_heads=1025), -2), (dict(head_dim=48), -2),
    (dict(head_dim=0), -2), (dict(head_dim=288), -2), (dict(ld_codes=2032), -1), (dict(ld_codes=2056), -1), (dict(ld_scales=124), -1), (dict(ld_scales=130), -1),
    (dict(ld_codes=1 << 32), -1), (dict(ld_codes=-2048), -1)])
def test_caches_that_are_refused(ctx, change, status):
    assert everything(ctx, cache(**change)) == {status}
    assert call("kv_attention_ws_bytes", ctx, cache(**change), seqs(), 5, 8) == 0


@pytest.mark.parametrize("change,status", [
    (dict(starts=None), -1), (dict(lengths=A + 2), -1), (dict(pages=None), -1), (dict(ld_pages=3), -1), (dict(count=-1), -1), (dict(max_pages=0), -2),
    (dict(max_new=-1), -1), (dict(max_length=-1), -1), (dict(count=0x7fffffff), -2), (dict(ld_pages=1 << 40), -1)])
def test_sequences_that_are_refused(ctx, change, status):
    assert everything(ctx, s=seqs(**change)) == {status}


def test_nothing_to_do(ctx):
    none = seqs(count=0, starts=None, lengths=None, pages=None, max_pages=0)
    assert everything(ctx, s=none) == {0}
    assert store(ctx, change=[(2, 0)]) == attend(ctx, change=[(2, 0)]) == load(ctx, change=[(2, 0)]) == 0
    assert load(ctx, change=[(3, None), (6, None)]) == 0
    assert call("rotate", ctx, turns(), None, 0, 2, 128, None, 256, 128, 1, 0, None, 256, 128) == 0


@pytest.mark.parametrize("at,value,status", [
    (2, -1, -1), (2, 1 << 31, -1), (3, None, -1), (3, A + 8, -1), (4, 252, -1), (4, -8, -1), (5, 1 << 40, -1), (6, None, -1), (7, 4, -1), (9, 2, -1), (9, -1, -1)])
def test_store_and_load_refuse(ctx, at, value, status):
    assert store(ctx, change=[(at, value)]) == status
    if not (at in (3, 6) and value is None):
        assert load(ctx, change=[(at, value)]) == status
    if at == 4:
        assert load(ctx, change=[(at, 120)]) == -1                       # rows in each other
        assert store(ctx, change=[(at, 0)]) == sb.ERR_HIP                # one row for all is fine to read


def test_store_refuses_rotations(ctx):
    good = dict(rotary=turns(), positions=A, q=A, q_heads=8, q_out=A + 4096)
    for k, status in ((dict(rotary=None), -1), (dict(rotary=turns(turns=None)), -1), (dict(rotary=turns(pairs=65)), -2), (dict(rotary=turns(pairs=0)), -2),
                      (dict(rotary=turns(interleaved=2)), -1), (dict(rotary=turns(amplitude=math.inf)), -1), (dict(q=None), -1), (dict(q_out=None), -1),
                      (dict(q_heads=0), -2), (dict(positions=A + 1), -1), (dict(q=A + 4), -1), (dict(q_out=A, change=[(17, 520)]), -1),
                      (dict(change=[(13, 511)]), -1), (dict(change=[(18, 64)]), -1)):
        assert store(ctx, **{**good, **k}) == status, k


@pytest.mark.parametrize("at,value,status", [
    (2, -1, -1), (3, 7, -2), (3, 0, -2), (3, 65536, -2), (2, 1 << 28, -2), (4, None, -1), (4, A + 2, -1), (5, 1020, -1), (7, 0.0, -1), (7, -1.0, -1), (7, math.nan, -1),
    (7, math.inf, -1), (7, 3e38, -1), (8, 2, -1), (9, -1, -1), (10, None, -1), (11, 64, -1), (12, 120, -1), (13, A + 2, -1)])
def test_attention_refuses(ctx, at, value, status):
    assert attend(ctx, change=[(at, value)]) == status
    assert attend(ctx, change=[(8, 0), (9, 5)]) == -1                    # a window needs an order
    assert attend(None) == -1


@pytest.mark.parametrize("at,value,status", [
    (0, None, -1), (0, turns(pairs=65), -2), (1, None, -1), (1, A + 2, -1), (2, -1, -1), (3, 0, -2), (4, 1, -2), (4, 257, -2), (5, None, -1), (5, A + 1, -1),
    (6, -1, -1), (8, 3, -1), (9, 2, -1), (10, None, -1), (11, 100, -1), (12, 64, -1)])
def test_rotate_refuses(ctx, at, value, status):
    args = [turns(), A, 3, 2, 128, A, 256, 128, 1, 0, A + 8192, 256, 128]
    args[at] = value
    assert call("rotate", ctx, *args) == status
    assert call("rotate", ctx, turns(), A, 3, 2, 128, A, 256, 128, 1, 0, A, 512, 128) == -1                # in place with other pitches
    assert call("rotate", None, turns(), A, 3, 2, 128, A, 256, 128, 1, 0, A, 256, 128) == -1


def test_turns_from_their_formulas():
    base, dims, context = 10000.0, 64, 4096
    f = [base ** (-2.0 * i / dims) / (2 * math.pi) for i in range(32)]
    close = lambda a, b: all(abs(x - y) <= 4 * 2.0 ** -53 * abs(y) for x, y in zip(a, b)) and len(a) == len(b)  # noqa: E731
    assert close(sb.rotary_turns(dims, base), f)
    assert close(sb.rotary_turns(dims, base, sb.ROTARY_LINEAR, factor=4.0), [x / 4 for x in f])
    def by_turns(x):
        n = context * x
        kept = 1.0 if n >= 4 else 0.0 if n <= 1 else (n - 1) / 3
        return kept * x + (1 - kept) * x / 8
    got = sb.rotary_turns(dims, base, sb.ROTARY_TURNS, factor=8.0, low=1.0, high=4.0, context=context)
    assert all(abs(a - by_turns(x)) < 1e-12 * x for a, x in zip(got, f)) and got[0] == pytest.approx(f[0]) and got[-1] == pytest.approx(f[-1] / 8)
    index = lambda n: dims * math.log(context / (2 * math.pi * n)) / (2 * math.log(base))  # noqa: E731
    a, b = math.floor(index(32)), math.ceil(index(1))
    got = sb.rotary_turns(dims, base, sb.ROTARY_INDEX, factor=8.0, low=1.0, high=32.0, context=context)
    for i, x in enumerate(f):
        kept = 1 - min(1.0, max(0.0, (i - a) / (b - a)))
        assert abs(got[i] - (kept * x + (1 - kept) * x / 8)) < 1e-12 * x
    for bad in (dict(base=1.0), dict(base=math.inf), dict(scaling=4), dict(scaling=1, factor=0.0), dict(scaling=2, low=2.0, high=2.0), dict(scaling=3, context=0.5),
                dict(scaling=2, low=0.0)):
        with pytest.raises(sb.SbitsError):
            sb.rotary_turns(64, **bad)
    with pytest.raises(sb.SbitsError):
        sb.rotary_turns(258)
    with pytest.raises(ValueError):
        sb.rotary_turns(7)


def test_binding_refuses(ctx):
    b = kv_plain.Batch([(2, 3), (1, 0)], 8, 2, 64)
    c, s, t = b.on(sb, dev="cpu")
    with pytest.raises(ValueError):
        sb.kv_cache(t[0], t[1], t[2], t[3], 128)
    with pytest.raises(ValueError):
        sb.kv_cache(t[0], t[1], t[2][:-1], t[3], 64)
    with pytest.raises(ValueError):
        sb.kv_cache(t[0].transpose(1, 2).contiguous().transpose(1, 2), *t[1:], 64)
    with pytest.raises(TypeError):
        sb.kv_cache(t[0].int(), *t[1:], 64)
    with pytest.raises(TypeError):
        sb.sequences(b.starts.long(), b.lengths, b.table)
    with pytest.raises(ValueError):
        sb.sequences(b.starts, b.lengths, b.table[:1])
    k = torch.zeros(3, 2, 64)
    with pytest.raises(TypeError):
        ctx.kv_store(c, s, k, k.bfloat16())
    with pytest.raises(TypeError):
        ctx.kv_store(c, s, k.half(), k.half())
    with pytest.raises(ValueError):
        ctx.kv_store(c, s, k, k, q=k, q_out=k)
    with pytest.raises(ValueError):
        ctx.kv_store(c, s, k[:, :1], k[:, :1])
    with pytest.raises(ValueError):
        ctx.kv_attention(c, s, k.bfloat16()[..., :32], k.bfloat16()[..., :32], None)
    with pytest.raises(TypeError):
        ctx.kv_attention(c, s, k, k, None)
    with pytest.raises(ValueError):
        ctx.kv_load(c, s, k, k[:2])
    with pytest.raises(TypeError):
        sb.rotary(torch.zeros(4))
    wide = torch.zeros(4, b.pages, 2, 8, 32, dtype=torch.uint8)                # layers' pages side by side
    scales = torch.zeros(4, b.pages, 2, 8, 4, dtype=torch.uint8)
    turned = sb.kv_cache(*(x.transpose(0, 1)[:, 1] for x in (wide, scales, wide, scales)), 64)
    assert turned.ld_codes == 2 * 8 * 32 and turned.pages == b.pages
    apart = sb.kv_cache(*(x.view(b.pages, 4, 2, 8, -1)[:, 1] for x in (wide, scales, wide, scales)), 64)
    assert apart.ld_codes == 4 * 2 * 8 * 32 and apart.ld_scales == 4 * 2 * 8 * 4
