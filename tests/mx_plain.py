"""Layers with 4-bit floating point weights from their definitions, in 64 bits on the CPU, and inputs for their tests."""
import math

import torch

GRID = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0, -0.0, -0.5, -1.0, -1.5, -2.0, -3.0, -4.0, -6.0], dtype=torch.float64)


def quantise(x):
    """Codes (one a byte) and bytes of x [rows, cols]."""
    b = x.double().reshape(x.shape[0], -1, 32)
    top = b.abs().amax(-1)
    fine = torch.isfinite(b).all(-1)
    power = torch.frexp(torch.where(fine, top, 1.0))[1] - 3
    power = torch.where(top == 0, -125, power).clamp(min=-125)
    size = (b.abs() * torch.exp2(-power.double())[..., None]).nan_to_num(posinf=9.0)
    # the nearest of the grid; of two the one whose code is even
    code = torch.zeros_like(size, dtype=torch.int64)
    least = size.clone()
    for k in range(1, 8):
        away = (size - GRID[k].item()).abs()
        nearer = (away < least) | (away == least) & (k % 2 == 0)
        code, least = torch.where(nearer, k, code), torch.where(nearer, away, least)
    code = torch.where(fine[..., None], code + 8 * torch.signbit(b), 0)
    return code.flatten(1).to(torch.uint8), torch.where(fine, power + 127, 255).to(torch.uint8)


def values(code, byte):
    scale = torch.where(byte == 255, math.nan, torch.exp2(byte.double() - 127))
    return (GRID.to(code.device)[code.long()].reshape(code.shape[0], -1, 32) * scale[..., None]).flatten(1)


def pack(code):
    return code[:, 0::2] | code[:, 1::2] << 4


def unpack(codes):
    return torch.stack((codes & 15, codes >> 4), -1).flatten(1)


def random_matrix(rows, cols, g, spread=3):
    """Codes and bytes, every code and some range of powers among them."""
    code = torch.randint(0, 16, (rows, cols), generator=g).to(torch.uint8)
    byte = torch.randint(120 - spread, 121 + spread, (rows, cols // 32), generator=g).to(torch.uint8)
    return code, byte


def stored(code, byte, dev, extra=0, junk=255):
    """(codes, scales, cols) on the device, pitches `extra` blocks longer than need be; what lies between holds junk."""
    rows, cols = code.shape
    c = torch.full((rows, cols // 2 + 16 * extra), junk, dtype=torch.uint8)
    c[:, :cols // 2] = pack(code)
    s = torch.full((rows, (cols // 32 + 3) // 4 * 4 + 4 * extra), junk, dtype=torch.uint8)
    s[:, :cols // 32] = byte
    return c.to(dev), s.to(dev), cols


def product(x, w, gated):
    """y, and how far sums in fp32 may be off (x, w in 64 bits): an addition may truncate, so each costs 2^-23 of the sums so far; a term
    takes part in at most as many as there are instructions along the row (16 columns or more to one), terms in an instruction, and
    partial sums to join, the last two below 256."""
    y = x @ w.T
    off = (x.abs() @ w.abs().T) * (x.shape[1] / 16 + 256) * 2.0 ** -23
    if gated:
        (a, u), (da, du) = y.chunk(2, 1), off.chunk(2, 1)
        s = a * torch.sigmoid(a)
        # the slope of silu is below 1.1; exp, a quotient and two products: 8 roundings
        return s * u, 1.1 * da * (u.abs() + du) + s.abs() * du + 8 * 2.0 ** -24 * (s * u).abs()
    return y, off


def route(r, logits, bias):
    x = logits.double()
    tokens, experts = x.shape
    fine = torch.isfinite(x)
    if r.scoring == 0:
        top = torch.where(fine, x, -math.inf).amax(-1, keepdim=True)
        e = torch.where(fine, torch.exp(x - torch.where(top > -math.inf, top, 0.0)), 0.0)
        p = e / e.sum(-1, keepdim=True).clamp(min=1e-300)
    else:
        p = torch.where(fine, torch.sigmoid(x), 0.0)
    score = p if bias is None else p + bias.double()
    if bias is not None:
        fine = fine & torch.isfinite(bias)
    ids = torch.full((tokens, r.top_k), -1, dtype=torch.int32)
    w = torch.zeros(tokens, r.top_k, dtype=torch.float64)
    each = experts // r.groups
    for t in range(tokens):
        left = [e for e in range(experts) if fine[t, e]]
        if r.groups > 1:
            worth = []
            for g in range(r.groups):
                s = sorted((score[t, e].item() for e in left if e // each == g), reverse=True)
                worth.append(-math.inf if not s else s[0] if r.group_score == 1 else sum(s[:2]))
            kept = sorted(range(r.groups), key=lambda g: (-worth[g], g))[:r.top_groups]
            left = [e for e in left if e // each in kept]
        key = x[t] if bias is None else score[t]
        left = sorted(left, key=lambda e: (-key[e].item(), e))[:r.top_k]
        ids[t, :len(left)] = torch.tensor(left, dtype=torch.int32)
        w[t, :len(left)] = p[t, left]
    if r.renormalize:
        total = w.sum(-1, keepdim=True)
        w = torch.where(total > 0, w / total, 0.0)
    return ids, w


def chosen_weights(r, x, ids):
    """The weights as a differentiable function of the logits (64 bits), the choice fixed."""
    fine = torch.isfinite(x)
    safe = torch.where(fine, x, -1e30)
    if r.renormalize and r.scoring == 0:        # (the sum over all experts cancels; in it, a gradient of 0 would be one of 1e-19)
        some = ids >= 0
        w = torch.softmax(torch.where(some, safe.gather(1, ids.clamp(min=0).long()), -1e30), -1)
        return torch.where(some, w, 0.0)
    p = torch.softmax(safe, -1) if r.scoring == 0 else torch.sigmoid(safe)
    some = ids >= 0
    w = torch.where(some, p.gather(1, ids.clamp(min=0).long()), 0.0)
    if r.renormalize:
        total = w.sum(-1, keepdim=True)
        w = w / torch.where(total > 0, total, 1.0)
    return w


def layer(r, logits, bias, x, up, down, four):
    """(ids, weights, out, how far out may be off); up, down: lists of matrices in 64 bits, x bf16, where the products are to be computed."""
    ids, w = route(r, logits, bias)
    xs = values(*quantise(x)) if four else x.double()
    tokens, hidden, d = x.shape[0], x.shape[1], 2.0 ** -7   # h: rounded to bf16, perhaps to the other side
    each, each_off = (torch.zeros(tokens, r.top_k, hidden, dtype=torch.float64, device=x.device) for _ in range(2))
    for e in range(r.experts):
        t, j = (i.to(x.device) for i in torch.nonzero(ids == e, as_tuple=True))
        if len(t) == 0:
            continue
        h, dh = product(xs[t], up[e], True)
        dh = dh + d * h.abs()
        h = h.to(torch.bfloat16).double()
        if four:
            q = values(*quantise(h))
            ends = [values(*quantise(h + s * dh)) for s in (-1, 1)]
            dh = torch.stack([(v - q).abs() for v in ends]).amax(0)
            h = q
        y, dy = product(h, down[e], False)
        each[t, j], each_off[t, j] = y, dy + dh @ down[e].abs().T + (2.0 ** -8 + 2.0 ** -22) * y.abs()
    weight = w.to(x.device)[..., None]
    out, off = (each * weight).sum(1), (each_off * weight).sum(1)
    return ids, w, out, off + 2.0 ** -8 * (out.abs() + off)
