"""A paged cache of keys and values in the microscaled form from its definitions, in 64 bits on the CPU, and inputs for its tests."""
import math
from fractions import Fraction

import torch

import mx_plain


def turn(x, positions, turns, interleaved, amplitude, back=False):
    """x [tokens, heads, dim] turned, in 64 bits, and how large the products were that an element is the sum of."""
    pairs = len(turns)
    # (whole turns come off in exact arithmetic: in 64 bits a position of 2^30 would leave an angle's error of 1e-7)
    part = [[float(q - round(q)) for q in (Fraction(t) * p for t in turns)] for p in positions.tolist()]
    angle = 2 * math.pi * torch.tensor(part, dtype=torch.float64).view(-1, 1, pairs)
    c, s = amplitude * torch.cos(angle), amplitude * torch.sin(angle) * (-1 if back else 1)
    x = x.double()
    out, size = x.clone(), x.abs()
    first = slice(0, 2 * pairs, 2) if interleaved else slice(0, pairs)
    second = slice(1, 2 * pairs, 2) if interleaved else slice(pairs, 2 * pairs)
    a, b = x[..., first], x[..., second]
    out[..., first], out[..., second] = a * c - b * s, b * c + a * s
    size[..., first], size[..., second] = (a * c).abs() + (b * s).abs(), (b * c).abs() + (a * s).abs()
    return out, size


def quantised(x):
    """x [.., dim] after rounding to the microscaled form: codes (one a byte) and bytes."""
    if x.numel() == 0:
        return torch.zeros(x.shape, dtype=torch.uint8), torch.zeros(*x.shape[:-1], x.shape[-1] // 32, dtype=torch.uint8)
    code, byte = mx_plain.quantise(x.reshape(-1, x.shape[-1]))
    return code.view(x.shape), byte.view(*x.shape[:-1], x.shape[-1] // 32)


def values(code, byte):
    if code.numel() == 0:
        return torch.zeros(code.shape, dtype=torch.float64)
    return mx_plain.values(code.reshape(-1, code.shape[-1]), byte.reshape(-1, byte.shape[-1])).view(code.shape)


class Batch:
    """Sequences of (new, past) tokens with their pages in any order; everything that belongs to no token holds junk."""

    def __init__(self, sizes, page, kv_heads, dim, seed=0, spread=3, lead=0, behind=0, spare=2, junk=255, extra_pages=1):
        g = torch.Generator().manual_seed(seed)
        self.sizes, self.page, self.kv_heads, self.dim, self.g = sizes, page, kv_heads, dim, g
        need = [-(-(n + p) // page) for n, p in sizes]
        self.pages = max(1, sum(need) + spare)
        order = torch.randperm(self.pages, generator=g).int()
        self.table = torch.full((len(sizes), max(1, max(need, default=1)) + extra_pages), -7, dtype=torch.int32)
        at = 0
        for b, n in enumerate(need):
            self.table[b, :n] = order[at:at + n]
            at += n
        starts = [lead]
        for n, _ in sizes:
            starts.append(starts[-1] + n)
        self.starts, self.lengths = torch.tensor(starts, dtype=torch.int32), torch.tensor([n + p for n, p in sizes], dtype=torch.int32)
        self.tokens = starts[-1] + behind
        self.row = (dim // 32 + 3) // 4 * 4
        self.codes = [torch.full((self.pages, kv_heads, page, dim // 2), junk, dtype=torch.uint8) for _ in "kv"]
        self.scales = [torch.full((self.pages, kv_heads, page, self.row), junk, dtype=torch.uint8) for _ in "kv"]
        for b, (n, p) in enumerate(sizes):
            for i in range(2):
                code, byte = mx_plain.random_matrix((n + p) * kv_heads, dim, g, spread)
                self.put(i, b, 0, code.view(n + p, kv_heads, dim), byte.view(n + p, kv_heads, dim // 32))

    def places(self, b, first, count):
        at = torch.arange(first, first + count)
        return self.table[b].long()[at // self.page], at % self.page

    def put(self, which, b, first, code, byte):
        page, at = self.places(b, first, len(code))
        self.codes[which][page, :, at] = mx_plain.pack(code.reshape(-1, self.dim)).view(*code.shape[:2], self.dim // 2)
        self.scales[which][page, :, at, :self.dim // 32] = byte

    def get(self, which, b, first, count):
        """Values [count, kv_heads, dim]."""
        page, at = self.places(b, first, count)
        code = mx_plain.unpack(self.codes[which][page, :, at].reshape(-1, self.dim // 2)).view(count, self.kv_heads, self.dim)
        return values(code, self.scales[which][page, :, at, :self.dim // 32])

    def positions(self):
        """Of the rows that belong to a sequence."""
        return torch.cat([torch.arange(p, p + n) for n, p in self.sizes]).int()

    def rows(self):
        """Which rows these are."""
        return torch.arange(int(self.starts[0]), int(self.starts[-1]))

    def on(self, sb, dev="cuda", **hints):
        """(cache, sequences) on the device; a list of buffers to look at."""
        t = [x.to(dev) for x in (self.codes[0], self.scales[0], self.codes[1], self.scales[1])]
        return sb.kv_cache(*t, self.dim), sb.sequences(self.starts.to(dev), self.lengths.to(dev), self.table.to(dev), **hints), t


def attention(batch, q, scale=None, causal=True, window=0, gone=()):
    """out and lse of the rows that belong to a sequence, in 64 bits, and how far they may be off.  gone: (sequence, page of it) that are not there.

    A score is a sum of dim products of up to 13 bits, taken in fp32 in some order: an addition may truncate, so each costs 2^-23 of the sums so far, and there are no
    more than dim / 32 * 4 of them plus those inside an instruction, below 256; q enters in four parts of 4 bits, less than 2^-18 of its block's largest
    value being left out (three parts: 2^-15).  With e the bound on a score (scaled), weights are off by e^(2 e) - 1 and, rounded to bf16 ahead of their product with v, by 2^-8
    each and by 2^-8 of the sum; powers of two, and the sums of weights, add 2^-20.  The output rounds
    once more.  A weight in fp16 is 2^9 times its size against a score
    that no weight counts more than 1 by; the smallest step is 2^-24: rounding to it costs 2^-25 / 2^9 of the key's v at most, against a sum of weights of 1 or more
    (where v is in bf16, powers below 2^-126 may count as 0, which costs less)."""
    dim, group = batch.dim, q.shape[1] // batch.kv_heads
    scale = dim ** -0.5 if scale is None else scale
    out, lse, off, off_lse = [], [], [], []
    row = int(batch.starts[0])
    for b, (n, p) in enumerate(batch.sizes):
        k, v = (batch.get(i, b, 0, n + p).transpose(0, 1).repeat_interleave(group, 0) for i in range(2))       # [heads, length, dim]
        x = q[row:row + n].double().transpose(0, 1)
        if n + p:                                                                # the bytes from 253 on: values beyond bf16's range
            page, place = batch.places(b, 0, n + p)
            far_out = (batch.scales[1][page, :, place, :dim // 32] >= 253).repeat_interleave(32, -1).transpose(0, 1).repeat_interleave(group, 0)
            v = torch.where(far_out, math.nan, v)
        row += n
        key, at = torch.arange(n + p)[None, :], torch.arange(p, p + n)[:, None]
        seen = torch.ones(n, n + p, dtype=torch.bool)
        if causal:
            seen = (key <= at) & ((key > at - window) if window else True)
        for s, page in gone:
            if s == b:
                seen = seen & (key // batch.page != page)
        t = scale * (x @ k.transpose(1, 2))
        largest = x.unflatten(-1, (-1, 32)).abs().amax(-1, keepdim=True).expand(*x.shape[:2], -1, 32).flatten(-2)
        far = scale * ((dim / 8 + 256) * 2.0 ** -23 * x.abs() + 2.0 ** -15 * largest) @ k.abs().transpose(1, 2)
        far = torch.where(seen, far, 0.0).amax(-1, keepdim=True) if n + p else far.sum(-1, keepdim=True)
        t = torch.where(seen, t, -math.inf)
        some = seen.any(-1)[None, :, None]
        w = torch.where(some, torch.softmax(t, -1), 0.0)
        v = torch.where(seen.any(0)[None, :, None], v, 0.0)                         # what no row sees takes no part
        y = torch.zeros(x.shape, dtype=torch.float64)
        size, least = torch.zeros_like(y), torch.zeros_like(y)
        for i in range(n):                                                       # (nor does it in a row that does not)
            u = torch.where(seen[i][None, :, None], v, 0.0)
            y[:, i] = (w[:, i, None] @ u)[:, 0]
            size[:, i] = (w[:, i, None] @ u.abs())[:, 0]
            least[:, i] = u.abs().sum(1)
        out.append(y.transpose(0, 1))
        off.append(((torch.expm1(2 * far.clamp(max=100.0)) + 2.0 ** -7 + 2.0 ** -20) * size + 2.0 ** -8 * y.abs() + 2.0 ** -34 * least).transpose(0, 1))
        lse.append(torch.logsumexp(t, -1).transpose(0, 1))
        off_lse.append((far[..., 0] + 2.0 ** -20 + 2.0 ** -23 * lse[-1].transpose(0, 1).abs()).nan_to_num(posinf=0.0).transpose(0, 1))
    return tuple(torch.cat(part) for part in (out, lse, off, off_lse))


def turns(dims, base=10000.0):
    return [base ** (-2.0 * i / dims) / (2 * math.pi) for i in range(dims // 2)]
