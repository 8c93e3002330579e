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


# ---- what a row does not see ------------------------------------------------------------------------
def scribble(b, which, page, at, g, junk):
    """Places of the cache, all heads of them, with other codes and bytes."""
    if len(page) == 0:
        return
    b.codes[which][page, :, at] = torch.randint(0, 256, (len(page), b.kv_heads, b.dim // 2), generator=g).to(torch.uint8)
    bytes_ = torch.full((len(page), b.kv_heads, b.row), junk) if junk >= 0 else torch.randint(0, 256, (len(page), b.kv_heads, b.row), generator=g)
    b.scales[which][page, :, at] = bytes_.to(torch.uint8)


def unused(b):
    """Places that no sequence has."""
    free = torch.ones(b.pages, b.page, dtype=torch.bool)
    for s in range(len(b.sizes)):
        page, at = b.places(s, 0, int(b.lengths[s]))
        free[page, at] = False
    return free.nonzero(as_tuple=True)


SEEN = [[(1, 0), (1, 62), (1, 63), (1, 200), (2, 1500)], [(9, 70), (16, 300), (5, 3)], [(150, 40), (70, 0)]]


@pytest.mark.parametrize("junk", [0, 2, 103, 120, 141, 215, 252, 253, 255, -1])
@pytest.mark.parametrize("sizes", SEEN)
@pytest.mark.parametrize("dim", [64, 96, 128, 160])
def test_places_of_no_token_do_not_change_a_bit(ctx, junk, sizes, dim):
    """Behind the last tokens, on pages of no sequence, on page 0, which stands in for pages that are not there: whatever these hold."""
    b = Batch(sizes, 16, 2, dim, seed=dim, junk=127, lead=1)
    b.table[0, -1] = b.pages + 5
    q = queries(b, 4)
    want = attend(ctx, b, q)
    g = torch.Generator().manual_seed(junk + 2)
    for which in range(2):
        scribble(b, which, *unused(b), g, junk)
    for x, y in zip(attend(ctx, b, q), want):
        assert torch.equal(x, y)
    check(ctx, b, q)


@pytest.mark.parametrize("junk", [2, 100, 150, 215, 250, 255, -1])
@pytest.mark.parametrize("sizes", SEEN[1:])
@pytest.mark.parametrize("window", [0, 30])
@pytest.mark.parametrize("dim", [128, 96])
def test_hidden_keys_and_other_rows_do_not_change_a_bit(ctx, junk, sizes, window, dim):
    """Later tokens, with other keys, values and queries; and tokens ahead of all windows of the rows that are looked at."""
    b = Batch(sizes, 16, 1, dim, seed=dim + window)
    q = queries(b, 3)
    want = attend(ctx, b, q, window=window)
    g = torch.Generator().manual_seed(junk + 2)
    keep = []                                                    # rows from one on, up to one
    for s, (n, past) in enumerate(sizes):
        first, last = n // 3 if window else 0, n // 3 + (n + 2) // 3
        page, at = b.places(s, past + last, n - last)
        for which in range(2):
            scribble(b, which, page, at, g, junk)
        ahead = max(0, past + first - window + 1) if window else 0
        page, at = b.places(s, 0, ahead)
        for which in range(2):
            scribble(b, which, page, at, g, junk)
        keep.append(torch.arange(int(b.starts[s]) + first, int(b.starts[s]) + last))
    keep = torch.cat(keep)
    others = torch.ones(b.tokens, dtype=torch.bool)
    others[keep] = False
    q[others] = (q[others].float() * 3.7).to(BF16).flip(-1)
    for x, y in zip(attend(ctx, b, q, window=window), want):
        assert torch.equal(x[keep], y[keep])
    if 0 <= junk <= 215:                                         # (of larger keys scores leave fp32)
        check(ctx, b, q, window=window)


# ---- scores far from 0 -----------------------------------------------------------------------------
@pytest.mark.parametrize("power", [16, 19, 20, 21, 22, 23, 24, 25, 27, 30, 40, 60])
@pytest.mark.parametrize("sign", [1, -1])
@pytest.mark.parametrize("sizes", [[(1, 700), (3, 100)], [(100, 300)]])
@pytest.mark.parametrize("scale", [1.0, 0.7])
def test_scores_far_from_zero(ctx, power, sign, sizes, scale):
    """Scores that are whole multiples of 2^power, exact in 32 bits: only keys with the largest one count (the next is e^20000 times less), alike."""
    b = Batch(sizes, 16, 1, 64, seed=power)
    g = torch.Generator().manual_seed(power)
    for s, (n, past) in enumerate(sizes):
        page, at = b.places(s, 0, n + past)
        b.codes[0][page, :, at] = 0
        b.codes[0][page, 0, at, 0] = torch.randint(0, 8, (n + past,), generator=g).to(torch.uint8)          # an element of k: 0 .. 6
        b.scales[0][page, :, at] = 127
    q = torch.zeros(b.tokens, 2, 64, dtype=BF16)
    q[:, 0, 0], q[:, 1, 0] = sign * 2.0 ** power, sign * 1.5 * 2.0 ** power
    out, sums = attend(ctx, b, q, scale=scale)
    for s, (n, past) in enumerate(sizes):
        at, k, v = kv_tight.sequence(b, s)
        for i in range(n):
            seen = slice(0, past + i + 1)
            t = sign * k[0, seen, 0]
            best = t == t.max()
            want = v[0, seen][best].mean(0)
            for h, f in enumerate((1.0, 1.5)):
                row = int(b.starts[s]) + i
                # weights are alike, 2^9 times a power of the score's rounding: fp16 rounds them by 2^-11 of their size, which their sum does not have; then a product and bf16
                assert ((out[row, h].double() - want).abs() <= 2.0 ** -8 * want.abs() + (2.0 ** -11 + 2.0 ** -18) * v[0, seen][best].abs().mean(0)).all()
                lse = scale * f * 2.0 ** power * float(t.max()) + math.log(int(best.sum()))
                assert abs(float(sums[row, h]) - lse) <= 2.0 ** -20 * max(1.0, abs(lse))


# ---- large values ------------------------------------------------------------------------------------
def peaked(b, seed, others=0):
    """k of which only one element is not 0: code 7 (6) for one key in 997, `others` else."""
    for s in range(len(b.sizes)):
        page, at = b.places(s, 0, int(b.lengths[s]))
        b.codes[0][page, :, at] = 0
        code = torch.full((len(page),), others)
        code[seed % 13::997] = 7
        b.codes[0][page, 0, at, 0] = code.to(torch.uint8)
        b.scales[0][page, :, at] = 127


@pytest.mark.parametrize("byte", [199, 200, 209, 210, 230, 250])
@pytest.mark.parametrize("sizes", [[(1, 4000), (2, 2500)], [(100, 3000)]])
@pytest.mark.parametrize("dim", [64, 128, 160])
def test_large_values_of_one_block_leave_the_others_as_they_are(ctx, byte, sizes, dim):
    """A key of a sequence's first with large values in one block; most of the weight lies on thousands of keys behind it, each 2^-10 of the largest."""
    b = Batch(sizes, 16, 1, dim, seed=byte)
    peaked(b, byte)
    b.codes[1] &= 0x77                                           # (no signs: an output is as large as what it is a sum of)
    for s in range(len(sizes)):
        page, at = b.places(s, 3, 1)
        b.scales[1][page, 0, at, 1] = byte
    q = torch.zeros(b.tokens, 2, dim, dtype=BF16)
    q[:, :, 0] = 1.0
    check(ctx, b, q, scale=1.2)
    check(ctx, b, q, scale=1.2, lse=False)


@pytest.mark.parametrize("byte", [199, 205, 240, 252])
@pytest.mark.parametrize("sizes", [[(1, 9000), (2, 6000)], [(100, 9000)]])
def test_means_of_thousands_of_the_largest_values_are_finite(ctx, byte, sizes):
    """Equal scores, so that each key counts; some elements with the largest value in all keys, some with both signs of it."""
    b = Batch(sizes, 64, 1, 64, seed=byte)
    b.scales[1][:] = byte
    b.codes[1][..., :8] = 0x77
    b.codes[1][..., 8:12] = 0x7f
    q = torch.zeros(b.tokens, 2, 64, dtype=BF16)
    out, _ = check(ctx, b, q)
    assert torch.isfinite(out).all() and (out[..., :16] == 6.0 * 2.0 ** (byte - 127)).all()
    check(ctx, b, queries(b, 2), scale=0.3)


# ---- each key by itself --------------------------------------------------------------------------------
@pytest.mark.parametrize("sizes,kv_heads,group,page,dim,window", [
    ([(1, 5000)], 1, 4, 64, 128, 0), ([(1, 5000)], 2, 1, 8, 64, 0), ([(17, 3000), (1, 9)], 1, 2, 16, 128, 0), ([(17, 3000), (1, 9)], 2, 4, 32, 96, 700),
    ([(3, 4000), (1, 63), (5, 1100), (2, 1023), (1, 0), (16, 2047)], 3, 1, 16, 160, 0), ([(1, 20000)], 1, 8, 256, 256, 0), ([(1, 9000)], 1, 16, 64, 224, 5000),
    ([(100, 5000)], 1, 2, 64, 128, 0), ([(100, 5000), (40, 3000), (1, 800)], 2, 2, 16, 64, 0), ([(65, 7000)], 1, 1, 128, 192, 0), ([(129, 2000)], 1, 1, 8, 32, 1500),
    ([(200, 0), (70, 60)], 2, 3, 64, 96, 33), ([(3, 9000), (1, 63), (5, 1100), (1, 5), (16, 2047)], 2, 1, 32, 64, 800), ([(1, 1000 + 7 * i) for i in range(40)], 1, 2, 16, 64, 0)])
@pytest.mark.parametrize("causal", [True, False])
def test_each_key_by_itself(ctx, sizes, kv_heads, group, page, dim, window, causal):
    """Outputs that count keys: one that is lost, taken twice or multiplied with another's weight is outside of the bound (see kv_tight.Counted)."""
    window = window if causal else 0
    c = kv_tight.Counted(Batch(sizes, page, kv_heads, dim, seed=dim, lead=1), kv_heads * group)
    want = c.expected(causal, window)
    rows = c.b.rows()
    for hints in ((), dict(max_new=max(n for n, _ in sizes), max_length=max(n + p for n, p in sizes)), dict(max_new=1, max_length=1)):
        for lse in (True, False):
            out, sums = attend(ctx, c.b, c.q, lse, hints, scale=c.scale, causal=causal, window=window)
            got = out[rows].double()
            assert ((got - want).abs() <= c.bound(want)).all(), float(((got - want).abs() / c.bound(want).clamp(min=1e-30)).max())
            if lse:                                              # an element's share of the sum, in all elements together, is all of it
                total = torch.tensor([float(sum(2.0 ** (k % 3) for k in range(max(0, p + i + 1 - window) if window else 0, p + i + 1 if causal else n + p)))
                                      for n, p in sizes for i in range(n)], dtype=torch.float64)
                assert ((sums[rows].double() - torch.log(total)[:, None]).abs() <= 2.0 ** -18).all()


# ---- bytes read back -----------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", [BF16, torch.float32])
def test_all_bytes_and_codes_read_back(ctx, dtype):
    """Each byte with each code: 255 is NaN, values above the type's range are infinite, bytes below 2 give subnormals, in bf16 rounded below 2^-133."""
    b = Batch([(256, 0)], 64, 1, 32, seed=1)
    page, at = b.places(0, 0, 256)
    b.codes[0][page, 0, at] = (torch.arange(16).repeat(2)[0::2] | torch.arange(16).repeat(2)[1::2] << 4).to(torch.uint8)
    b.scales[0][page, 0, at, 0] = torch.arange(256).to(torch.uint8)
    cache, seqs, _ = b.on(sb)
    out = torch.zeros(256, 1, 32, dtype=dtype, device="cuda")
    ctx.kv_load(cache, seqs, out, None)
    grid = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], dtype=torch.float64)
    grid = torch.cat([grid, -grid])[torch.arange(16).repeat(2)]
    want = grid[None] * torch.tensor([2.0 ** (e - 127) for e in range(255)], dtype=torch.float64)[:, None]
    got = out.cpu()[:, 0]
    assert torch.isnan(got[255]).all()
    assert torch.equal(got[:255], want.to(dtype))                # (both roundings to nearest even, and to infinity)


# ---- beyond fp32 -----------------------------------------------------------------------------------------
@pytest.mark.parametrize("sizes", [[(1, 300)], [(100, 60)]])
def test_scores_beyond_fp32(ctx, sizes):
    """Above the range: NaN for the rows that see the key; below it: as if it were not there."""
    b = Batch(sizes, 16, 1, 64, seed=4)
    n, past = sizes[0]
    q = queries(b, 2)
    q[:, :, 0] = 2.0 ** 20
    page, at = b.places(0, 0, n + past)
    b.codes[0][page, 0, at, 0] &= 0xf0                           # k's first element: 0
    want = attend(ctx, b, q)
    key = past // 2
    b.codes[0][page[key], 0, at[key]] = 0
    for code in (0xf, 0x7):                                      # -6 and 6 times 2^125, and 2^20 in q
        b.codes[0][page[key], 0, at[key], 0] = code
        b.scales[0][page[key], 0, at[key], 0] = 252
        out, sums = attend(ctx, b, q)
        if code == 0x7:
            assert torch.isnan(out).all()
            continue
        b2 = Batch(sizes, 16, 1, 64, seed=4)
        b2.codes, b2.scales = [c.clone() for c in b.codes], [s.clone() for s in b.scales]
        b2.codes[0][page[key], 0, at[key]] = 0
        b2.codes[0][page[key], 0, at[key], 0], b2.scales[0][page[key], 0, at[key], 0] = 0xf, 140      # -6 * 2^13 * 2^20 / 8: e^-6e9
        other, other_sums = attend(ctx, b2, q)
        assert torch.equal(out, other) and torch.equal(sums, other_sums)
        assert torch.isfinite(out).all() and want[0].shape == out.shape


def test_keys_turned_beyond_fp32_are_its_largest_number(ctx):
    b = Batch([(1, 0)], 16, 1, 32)
    cache, seqs, buffers = b.on(sb)
    k = torch.full((1, 1, 32), 3e38)
    k[..., 16:] = -3e38
    turn = torch.full((16,), 0.125, dtype=torch.float64, device="cuda")                  # at position 1 an eighth of a turn: (a, -a) to (1.41 a, 0)
    ctx.kv_store(cache, seqs, k.cuda(), k.cuda(), rotary=sb.rotary(turn), positions=torch.ones(1, dtype=torch.int32, device="cuda"))
    out = torch.zeros(1, 1, 32, device="cuda")
    ctx.kv_load(cache, seqs, out, None)
    assert (out[..., :16] == 6.0 * 2.0 ** 125).all() and (out[..., 16:].abs() <= 2.0 ** 123).all()
