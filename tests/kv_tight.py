"""Attention to the microscaled cache in 64 bits from what lies in its buffers (pages by the table, lengths and starts as they are), with bounds that count each rounding
of the kernels once, and inputs for which a single lost or misplaced key is far outside of them."""
import math

import torch

import kv_plain
import mx_plain


def sequence(b, s):
    """Which positions of sequence s are there, and their keys and values [kv_heads, positions, dim] (values with bytes from 253 on: NaN)."""
    length = max(int(b.lengths[s]), 0)
    at = torch.arange(min(length, b.table.shape[1] * b.page))
    page = b.table[s].long()[at // b.page] if len(at) else at
    at, page = at[(page >= 0) & (page < b.pages)], page[(page >= 0) & (page < b.pages)]
    out = []
    for i in range(2):
        code = mx_plain.unpack(b.codes[i][page, :, at % b.page].reshape(-1, b.dim // 2)).view(len(at), b.kv_heads, b.dim)
        byte = b.scales[i][page, :, at % b.page, :b.dim // 32]
        x = kv_plain.values(code, byte)
        if i:
            x = torch.where((byte >= 253).repeat_interleave(32, -1), math.nan, x)
        out.append(x.transpose(0, 1))
    return at, *out


def attention(b, q, scale=None, causal=True, window=0, terms=3):
    """out and lse [rows of sequences, heads, ..] and how far they may be off.

    A score: sums in fp32 of products that are exact, each addition off by 2^-23 of the magnitudes' sum, of which there are no more than terms * dim / 32 and 256 inside
    instructions; of q what the terms leave out, 2^-15 of its block's largest value with three of them and 2^-18 with four.  A weight: the power of two is off by a unit in the last
    place, 2^-23; its argument, 9 to 15 and the largest score's size, by half a unit of numbers below 16, 2^-21, and 2^-23 of that size; rounded to fp16 2^-11 and, where it is small, by 2^-25 against a
    sum of 2^9.  Sums of weights: 2^-24 for each key, and for what joins them; of products, 16 or 32 at a time, 2^-23 each.  The output: bf16, 2^-8.  Below 2^-126 steps are no longer relative: bf16 rounds by up to
    2^-134, and a product of a weight with v that the matrix cores may count as 0 is below 2^-126, against a sum of weights of 2^9, or where the row sees values from 2^73 on, of 2^-31."""
    dim, group = b.dim, q.shape[1] // b.kv_heads
    scale = dim ** -0.5 if scale is None else scale
    parts = []
    for s in range(len(b.lengths)):
        first, end = int(b.starts[s]), int(b.starts[s + 1])
        key, k, v = sequence(b, s)
        at = int(b.lengths[s]) - end + torch.arange(first, end)[:, None]
        seen = torch.ones(end - first, len(key), dtype=torch.bool)
        if causal:
            seen = (key <= at) & (key > at - window) if window else key <= at
        x = q[first:end].double().unflatten(1, (b.kv_heads, group))                 # [rows, kv_heads, group, dim]
        t = scale * torch.einsum("nhgd,hkd->nhgk", x, k)
        largest = x.unflatten(-1, (-1, 32)).abs().amax(-1, keepdim=True).expand(*x.shape[:-1], -1, 32).flatten(-2)
        far = scale * torch.einsum("nhgd,hkd->nhgk", (terms * dim / 32 + 256) * 2.0 ** -23 * x.abs() + 2.0 ** (-15 if terms == 3 else -18) * largest, k.abs())
        hide = ~seen[:, None, None, :]
        t, far = t.masked_fill(hide, -math.inf), far.masked_fill(hide, 0.0)
        size_t = t.masked_fill(hide, 0.0).abs()
        far, size_t = (z.amax(-1, keepdim=True) if len(key) else z.sum(-1, keepdim=True) for z in (far, size_t))
        lse = torch.logsumexp(t, -1)
        w = torch.where(seen.any(-1)[:, None, None, None], torch.softmax(t, -1), 0.0)
        y, size, least = (torch.zeros_like(x) for _ in range(3))
        largest_v = torch.zeros(end - first, b.kv_heads, dtype=torch.float64)
        for i in range(end - first):                                              # (what a row does not see takes no part, whatever it is)
            u = v.masked_fill(~seen[i][None, :, None], 0.0)
            y[i], size[i] = torch.einsum("hgk,hkd->hgd", w[i], u), torch.einsum("hgk,hkd->hgd", w[i], u.abs())
            least[i] = u.abs().sum(1)[:, None]
            if len(key):
                largest_v[i] = u.abs().nan_to_num(nan=0.0).amax((1, 2))
        power = (3 + size_t) * 2.0 ** -22 + (len(key) + 64) * 2.0 ** -24
        lost = 2.0 ** -134 + len(key) * torch.where((largest_v >= 2.0 ** 72)[:, :, None, None], 2.0 ** -95, 2.0 ** -135)
        off = (torch.expm1(2 * (far + power).clamp(max=100.0)) + 2.0 ** -11 + (len(key) / 16 + 64) * 2.0 ** -23) * size + 2.0 ** -8 * y.abs() + 2.0 ** -34 * least \
            + lost
        off_lse = (far + power)[..., 0] + 2.0 ** -22 * (1 + lse.abs().nan_to_num(posinf=0.0))
        parts.append([z.flatten(1, 2) for z in (y, lse, off, off_lse)])
    return tuple(torch.cat(p) for p in zip(*parts))


class Counted:
    """A batch whose outputs show each key by itself: key j's value is 1 in the elements d with d % period == j % period, 0 in others, and its weight one of three powers of two
    (by j % 3), so that an element is a sum of few weights, of which the least is far above what the output's rounding takes.  Scores are whole multiples of log 2."""

    def __init__(self, batch, heads):
        self.b, dim = batch, batch.dim
        for s, length in enumerate(batch.lengths.tolist()):
            key = torch.arange(length)
            page, at = batch.places(s, 0, length)
            # k: the first element 0, 1 or 2 (codes 0, 2, 4), v: code 2 is 1
            code = torch.zeros(length, batch.kv_heads, dim, dtype=torch.uint8)
            code[:, :, 0] = (2 * (key % 3))[:, None].to(torch.uint8)
            one = 2 * (torch.arange(dim)[None, None, :] == self.element(key, batch.kv_heads)[..., None]).to(torch.uint8)
            byte = torch.full((length, batch.kv_heads, dim // 32), 127, dtype=torch.uint8)
            batch.put(0, s, 0, code, byte)
            batch.put(1, s, 0, one, byte)
        self.q = torch.zeros(batch.tokens, heads, dim, dtype=torch.bfloat16)
        self.q[:, :, 0] = 1.0
        self.scale = math.log(2.0)

    def element(self, key, kv_heads):
        return (key[:, None] + 7 * torch.arange(kv_heads)) % self.b.dim

    def expected(self, causal=True, window=0, lost=()):
        """Sums of weights by element and their quotient, without the keys in `lost` (of each sequence; to see what that makes)."""
        b, group = self.b, self.q.shape[1] // self.b.kv_heads
        out = []
        for s, (n, past) in enumerate(b.sizes):
            key = torch.arange(n + past)
            w = 2.0 ** (key % 3).double()
            for i in range(n):
                last = past + i + 1 if causal else n + past
                first = max(0, last - window) if window else 0
                seen = (key >= first) & (key < last)
                total = (w * seen).sum()
                kept = seen.clone()
                kept[[k for k in lost if k < len(key)]] = False
                y = torch.zeros(b.kv_heads, b.dim, dtype=torch.float64)
                for h in range(b.kv_heads):
                    y[h].index_add_(0, self.element(key, b.kv_heads)[:, h], w * kept)
                out.append((y / total).repeat_interleave(group, 0))
        return torch.stack(out)

    @staticmethod
    def bound(want):
        """Weights: their power's argument is off by 2^-20 (scores below 2 in magnitude, and what is taken off, below 32), fp16 rounds by 2^-11; the output by 2^-8."""
        return want * (2.0 ** -8 + 2.0 ** -11 + 2.0 ** -18)
