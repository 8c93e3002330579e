"""Workloads on which the operators of layers with 4-bit floating point weights are measured.

  quantise   a tensor to the microscaled 4-bit form (32 elements share a power of two) and the values it then stands for
  product    activations, in 16 bits or quantised to 4, times a matrix in that form; plain or gated (silu(g) * u)
  route      the choice of experts for each token, with weights; or the gradient of those weights with respect to the logits
  experts    a whole layer of experts: routing, lists, both products, the weighted sum

`own` chooses between the library's calls and the operators' plain forms in elementary torch operations.
A case is a dict of plain values; `listed()` holds named sizes, `draw()` gives further ones of the same ranges.
"""
from __future__ import annotations

import math

import torch

own = False

GRID = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0, -0.0, -0.5, -1.0, -1.5, -2.0, -3.0, -4.0, -6.0)
MOST_ELEMENTS = 8192 * 14336             # of the largest listed quantisation
MOST_FLOPS = 2 * 8192 * 14336 * 4096     # of the largest listed product
MOST_WEIGHTS = 32 * 3 * 4096 * 2048      # of the largest listed set of experts
MOST_LAYER_FLOPS = 6 * 4096 * 4 * 4096 * 2048
MOST_SCORES = 16384 * 256                # of the largest listed routing


def listed():
    return [
        # ---- quantise: the state of one token ahead of a projection of the 8B shape --------------------
        {"name": "quantise_token", "kind": "quantise", "rows": 1, "cols": 4096, "type": "bf16", "pad": 0},
        # the MLP activations of a prefill of 8192 tokens of the 8B shape
        {"name": "quantise_prefill", "kind": "quantise", "rows": 8192, "cols": 14336, "type": "bf16", "pad": 0},
        # sums of another product, in fp32, as rows of a wider buffer; blocks that do not fill a tile
        {"name": "quantise_ragged_f32", "kind": "quantise", "rows": 1001, "cols": 1056, "type": "fp32", "pad": 96},
        # ---- product: one token through the gate projection of the 8B shape ----------------------------
        {"name": "product_token", "kind": "product", "batch": 1, "rows": 14336, "cols": 4096, "x": 16, "gated": False, "out": "fp32"},
        # decoding for an odd number of sequences through the down projection
        {"name": "product_decode_b37", "kind": "product", "batch": 37, "rows": 4096, "cols": 14336, "x": 16, "gated": False, "out": "bf16"},
        # a chunk of a prompt through gate and up with the activation behind them, activations in 16 bits
        {"name": "product_chunk_gated", "kind": "product", "batch": 1000, "rows": 14336, "cols": 4096, "x": 16, "gated": True, "out": "bf16"},
        # a long prefill with the activations in 4 bits, too
        {"name": "product_prefill_4bit", "kind": "product", "batch": 8192, "rows": 14336, "cols": 4096, "x": 4, "gated": False, "out": "bf16"},
        # ---- route: one token, the latency of a call ---------------------------------------------------
        {"name": "route_token", "kind": "route", "tokens": 1, "experts": 64, "top_k": 8, "score": "softmax", "bias": False, "groups": 1,
         "top_groups": 1, "renormalize": True, "type": "fp32", "backward": False},
        # a prefill with many experts: sigmoid scores, a bias for balance, the best four of eight groups
        {"name": "route_prefill", "kind": "route", "tokens": 16384, "experts": 256, "top_k": 8, "score": "sigmoid", "bias": True, "groups": 8,
         "top_groups": 4, "renormalize": True, "type": "fp32", "backward": False},
        # the router's gradient on a training batch
        {"name": "route_backward", "kind": "route", "tokens": 16384, "experts": 128, "top_k": 8, "score": "softmax", "bias": False, "groups": 1,
         "top_groups": 1, "renormalize": False, "type": "bf16", "backward": True},
        # ---- experts: decoding for 16 sequences, most experts with a row or two ------------------------
        {"name": "experts_decode", "kind": "experts", "tokens": 16, "experts": 64, "top_k": 8, "score": "softmax", "bias": False, "groups": 1,
         "top_groups": 1, "renormalize": True, "type": "fp32", "hidden": 2048, "inner": 1024, "x": 16},
        # a prefill through large experts, activations in 4 bits
        {"name": "experts_prefill", "kind": "experts", "tokens": 4096, "experts": 32, "top_k": 4, "score": "sigmoid", "bias": True, "groups": 4,
         "top_groups": 2, "renormalize": True, "type": "bf16", "hidden": 4096, "inner": 2048, "x": 4},
    ]


# ---- drawing cases ---------------------------------------------------------------------------------
def _log(rng, lo, hi, step=1):
    """A multiple of `step` in lo..hi, spread over the logarithm."""
    v = math.exp(rng.uniform(math.log(lo), math.log(max(lo, hi) + 0.99)))
    return max(step, int(v) // step * step)


def _router(rng, experts):
    groups = rng.choice([1, 1, 2, 4, 8])
    top_groups = rng.randint(1, groups)
    top_k = min(rng.choice([1, 2, 4, 6, 8]), experts // groups * top_groups)
    return {"experts": experts, "top_k": top_k, "score": rng.choice(["softmax", "sigmoid"]), "bias": rng.random() < 0.5, "groups": groups,
            "top_groups": top_groups, "renormalize": rng.random() < 0.7, "type": rng.choice(["fp32", "bf16"])}


def draw(rng):
    kind = rng.choice(["quantise", "product", "product", "product", "route", "experts", "experts"])
    if kind == "quantise":
        cols = _log(rng, 32, 28672, 32)
        return {"kind": kind, "rows": _log(rng, 1, min(16384, MOST_ELEMENTS // cols)), "cols": cols, "type": rng.choice(["bf16", "fp32"]),
                "pad": rng.choice([0, 0, 8, 160])}
    if kind == "product":
        rows, cols, gated = _log(rng, 250, 28672), _log(rng, 256, 14336, 32), rng.random() < 0.3
        most = MOST_FLOPS // (2 * rows * cols * (2 if gated else 1))
        return {"kind": kind, "batch": _log(rng, 1, max(1, min(8192, most))), "rows": rows, "cols": cols, "x": rng.choice([16, 16, 4]), "gated": gated,
                "out": rng.choice(["fp32", "bf16"])}
    if kind == "route":
        experts = rng.choice([8, 16, 24, 64, 72, 128, 160, 256])
        backward = rng.random() < 0.35
        return {"kind": kind, "tokens": _log(rng, 1, min(32768, MOST_SCORES // experts)), **_router(rng, experts), "backward": backward}
    experts = rng.choice([8, 16, 32, 64, 128])
    hidden = _log(rng, 512, 4096, 32)
    inner = _log(rng, 256, min(4096, MOST_WEIGHTS // (experts * 3 * hidden)), 32)
    case = {"kind": kind, "tokens": 0, **_router(rng, experts), "hidden": hidden, "inner": inner, "x": rng.choice([16, 4])}
    case["tokens"] = _log(rng, 1, max(1, min(4096, MOST_LAYER_FLOPS // (6 * case["top_k"] * hidden * inner))))
    return case


# ---- inputs ----------------------------------------------------------------------------------------
def _generator(seed, part):
    return torch.Generator(device="cuda").manual_seed(seed * 1000003 + part)


def _type(name):
    return torch.bfloat16 if name == "bf16" else torch.float32


def _activations(rows, cols, seed):
    """Hidden states: normal, with channels of ten times the size, as a residual stream has them."""
    g = _generator(seed, 1)
    x = torch.randn(rows, cols, generator=g, device="cuda")
    large = torch.rand(cols, generator=g, device="cuda") < 0.005
    return x.mul_(torch.where(large, 10.0, 1.0)).to(torch.bfloat16)


def _weights(rows, cols, seed, part):
    """A stored matrix: weights of heavy tails in the 4-bit form, made in pieces of some rows."""
    g = _generator(seed, part)
    codes = torch.empty(rows, cols // 2, dtype=torch.uint8, device="cuda")
    scales = torch.empty(rows, (cols // 32 + 3) // 4 * 4, dtype=torch.uint8, device="cuda").fill_(127)
    piece = max(1, (64 << 20) // cols)
    for at in range(0, rows, piece):
        w = torch.randn(min(piece, rows - at), cols, generator=g, device="cuda").mul_(0.02)
        w *= torch.rand(w.shape[0], 1, generator=g, device="cuda").mul_(2.0).exp_()
        code, byte = _quantise(w)
        codes[at:at + piece] = code[:, 0::2] | code[:, 1::2] << 4
        scales[at:at + piece, :cols // 32] = byte
    return codes, scales


def _logits(case, seed):
    """Scores of a router: some experts are liked more than others, a few tokens are padding, a few experts are masked."""
    g = _generator(seed, 5)
    tokens, experts = case["tokens"], case["experts"]
    like = torch.randn(experts, generator=g, device="cuda").mul_(0.5)
    logits = torch.randn(tokens, experts, generator=g, device="cuda").mul_(1.5).add_(like)
    hidden = torch.rand(tokens, experts, generator=g, device="cuda") < 0.01
    logits.masked_fill_(hidden, -math.inf)
    if tokens > 8:
        logits.masked_fill_(torch.rand(tokens, 1, generator=g, device="cuda") < 0.01, -math.inf)
    return logits.to(_type(case["type"])), torch.randn(experts, generator=g, device="cuda").mul_(0.02) if case["bias"] else None


def prepare(case, seed):
    kind = case["kind"]
    state = dict(case=case)
    if kind == "quantise":
        wide = _activations(case["rows"], case["cols"] + case["pad"], seed)
        if case["type"] == "fp32":
            wide = wide.float() + 1e-3 * torch.randn(wide.shape, generator=_generator(seed, 2), device="cuda")
        state["x"] = wide[:, :case["cols"]]
    elif kind == "product":
        state["x"] = _activations(case["batch"], case["cols"], seed)
        state["w"] = _weights(case["rows"] * (2 if case["gated"] else 1), case["cols"], seed, 3)
    else:
        state["logits"], state["bias"] = _logits(case, seed)
        if kind == "experts":
            state["x"] = _activations(case["tokens"], case["hidden"], seed)
            state["up"] = _weights(case["experts"] * 2 * case["inner"], case["hidden"], seed, 3)
            state["down"] = _weights(case["experts"] * case["hidden"], case["inner"], seed, 4)
        elif case["backward"]:
            state["ids"], _ = _route(case, state["logits"], state["bias"])
            state["d_weights"] = torch.randn(case["tokens"], case["top_k"], generator=_generator(seed, 6), device="cuda")
    return state


# ---- the plain forms -------------------------------------------------------------------------------
def _quantise(x):
    """Codes and the byte of each block's power of two, one code a byte."""
    blocks = x.float().unflatten(-1, (-1, 32))
    largest = blocks.abs().amax(-1)
    power = torch.frexp(largest)[1] - 3
    power = torch.where(largest == 0, -125, power).clamp_(min=-125).int()
    broken = ~torch.isfinite(largest)
    size = blocks.abs() * (127 - power << 23).view(torch.float32)[..., None]
    code = ((size > 0.25).to(torch.uint8) + (size >= 0.75) + (size > 1.25) + (size >= 1.75) + (size > 2.5) + (size >= 3.5) + (size > 5.0)
            + torch.signbit(blocks) * 8)
    code = torch.where(broken[..., None], 0, code).to(torch.uint8)
    return code.flatten(-2), torch.where(broken, 255, power + 127).to(torch.uint8)


def _values(code, byte):
    """What codes and bytes stand for."""
    grid = torch.tensor(GRID, device=code.device)
    scale = torch.where(byte == 255, math.nan, (byte.int() << 23).view(torch.float32))
    return (grid[code.int()].unflatten(-1, (-1, 32)) * scale[..., None]).flatten(-2)


def _stored(w, cols):
    codes, scales = w
    return _values(torch.stack((codes & 15, codes >> 4), -1).flatten(-2), scales[:, :cols // 32])


def _gate(y):
    g, u = y.chunk(2, -1)
    return g / (1 + torch.exp(-g)) * u


def _route(case, logits, bias):
    """The chosen experts, descending, -1 where none is left; and their weights."""
    logits = logits.float()
    fine = torch.isfinite(logits)
    wide = logits.double()
    if case["score"] == "softmax":
        top = torch.where(fine, wide, -math.inf).amax(-1, keepdim=True)
        e = torch.where(fine, torch.exp(wide - torch.where(torch.isfinite(top), top, 0.0)), 0.0)
        p = e / e.sum(-1, keepdim=True).clamp_(min=1e-300)
    else:
        p = torch.where(fine, 1 / (1 + torch.exp(-wide)), 0.0)
    score = p if bias is None else p + bias.double()
    order = wide if bias is None else score          # (the same order, but where scores round to the same)
    order = torch.where(fine, order, -math.inf)
    if case["groups"] > 1:
        inside = torch.where(fine, score, -math.inf).unflatten(-1, (case["groups"], -1))
        best = torch.sort(inside, dim=-1, descending=True)[0][..., :2]
        some = torch.isfinite(best[..., 0])
        group = torch.where(some, torch.where(torch.isfinite(best), best, 0.0).sum(-1), -math.inf)
        taken = torch.sort(group, dim=-1, descending=True, stable=True)[1][:, :case["top_groups"]]
        open_ = torch.zeros_like(group, dtype=torch.bool).scatter_(1, taken, True)
        order = torch.where(open_[..., None], order.unflatten(-1, (case["groups"], -1)), -math.inf).flatten(-2)
    chosen, ids = torch.sort(order, dim=-1, descending=True, stable=True)
    ids = ids[:, :case["top_k"]]
    some = torch.isfinite(chosen[:, :case["top_k"]])
    weights = torch.where(some, p.gather(1, ids), 0.0)
    if case["renormalize"]:
        total = weights.sum(-1, keepdim=True)
        weights = torch.where(total > 0, weights / total, 0.0)
    return torch.where(some, ids, -1).int(), weights.float()


def _route_backward(case, logits, ids, d_weights):
    logits = logits.float()
    fine = torch.isfinite(logits)
    if case["score"] == "softmax":
        top = torch.where(fine, logits, -math.inf).amax(-1, keepdim=True)
        e = torch.where(fine, torch.exp(logits - torch.where(torch.isfinite(top), top, 0.0)), 0.0)
        p = e / e.sum(-1, keepdim=True).clamp_(min=1e-30)
    else:
        p = torch.where(fine, 1 / (1 + torch.exp(-logits)), 0.0)
    some = ids >= 0
    at = torch.where(some, ids, 0).long()
    chosen = torch.where(some, p.gather(1, at), 0.0)
    g = torch.where(some, d_weights, 0.0)
    if case["renormalize"]:
        total = chosen.sum(-1, keepdim=True)
        share = torch.where(total > 0, chosen / total, 0.0)
        g = share * (g - (g * share).sum(-1, keepdim=True))
        if case["score"] == "sigmoid":
            g = g * (1 - chosen)
        return torch.zeros_like(p).scatter_add_(1, at, torch.where(some, g, 0.0))
    if case["score"] == "sigmoid":
        return torch.zeros_like(p).scatter_add_(1, at, torch.where(some, g * chosen * (1 - chosen), 0.0))
    spread = torch.zeros_like(p).scatter_add_(1, at, g)
    return p * (spread - (g * chosen).sum(-1, keepdim=True))


def _layer(state):
    """Rows by expert, as many for each as the fullest has; both products over all experts at once."""
    case = state["case"]
    experts, hidden, inner, k = case["experts"], case["hidden"], case["inner"], case["top_k"]
    ids, weights = _route(case, state["logits"], state["bias"])
    slot = ids.flatten().long()
    kept = torch.nonzero(slot >= 0).flatten()
    expert, at = torch.sort(slot[kept], stable=True)
    kept = kept[at]
    counts = (expert[:, None] == torch.arange(experts, device="cuda")).sum(0)
    place = torch.arange(len(kept), device="cuda") - (counts.cumsum(0) - counts)[expert]
    x = state["x"].float()
    if case["x"] == 4:
        x = _values(*_quantise(x))
    most = max(1, int(counts.max()))
    rows = torch.zeros(experts, most, hidden, device="cuda")
    rows[expert, place] = x[kept // k]
    y = torch.bmm(_stored(state["up"], hidden).view(experts, 2 * inner, hidden), rows.transpose(1, 2).contiguous())
    g, u = y.chunk(2, 1)
    h = (g / (1 + torch.exp(-g)) * u).to(torch.bfloat16).float()
    if case["x"] == 4:
        h = _values(*_quantise(h.transpose(1, 2))).transpose(1, 2).contiguous()
    y = torch.bmm(_stored(state["down"], inner).view(experts, hidden, inner), h)
    each = torch.zeros(case["tokens"] * k, hidden, device="cuda")
    each[kept] = y.transpose(1, 2)[expert, place].to(torch.bfloat16).float()
    out = (each.view(-1, k, hidden) * weights[..., None]).sum(1)
    return {"out": out.to(torch.bfloat16), "ids": ids, "weights": weights}


def _plain(state):
    case = state["case"]
    if case["kind"] == "quantise":
        code, byte = _quantise(state["x"])
        return {"values": _values(code, byte).to(torch.bfloat16), "scales": byte.view(torch.float8_e8m0fnu)}
    if case["kind"] == "product":
        x = state["x"].float()
        if case["x"] == 4:
            x = _values(*_quantise(x))
        y = torch.matmul(x, _stored(state["w"], case["cols"]).t())
        return (_gate(y) if case["gated"] else y).to(_type(case["out"]))
    if case["kind"] == "experts":
        return _layer(state)
    if case["backward"]:
        return _route_backward(case, state["logits"], state["ids"], state["d_weights"])
    return dict(zip(("ids", "weights"), _route(case, state["logits"], state["bias"])))


# ---- the library's calls ---------------------------------------------------------------------------
_program = {}


def _context():
    """What a program holds for all its calls: the context of its stream and a workspace that grows."""
    from paper_2602_17698_amd import binding as sb
    if "ctx" not in _program:
        _program["ctx"] = sb.Context(0, torch.cuda.current_stream().cuda_stream)
        _program["ws"] = torch.empty(1 << 20, dtype=torch.uint8, device="cuda")
    return sb, _program["ctx"]


def _workspace(size):
    if _program["ws"].numel() < size:
        _program["ws"] = torch.empty(size, dtype=torch.uint8, device="cuda")
    return _program["ws"]


def _router_of(sb, case):
    return sb.Router(experts=case["experts"], top_k=case["top_k"], scoring=sb.ROUTE_SOFTMAX if case["score"] == "softmax" else sb.ROUTE_SIGMOID,
                     groups=case["groups"], top_groups=case["top_groups"], group_score=sb.ROUTE_GROUP_TOP2, renormalize=case["renormalize"])


def _own(state):
    case = state["case"]
    sb, ctx = _context()
    new = lambda *size, dtype: torch.empty(*size, dtype=dtype, device="cuda")  # noqa: E731
    if case["kind"] == "quantise":
        rows, cols = case["rows"], case["cols"]
        q = sb.mx(new(rows, cols // 2, dtype=torch.uint8), new(rows, sb.mx_scale_pitch(cols), dtype=torch.uint8), cols)
        values = new(rows, cols, dtype=torch.bfloat16)
        ctx.mx_quantize(state["x"], q, values)
        return {"values": values, "scales": q.scales_tensor[:, :cols // 32].view(torch.float8_e8m0fnu)}
    if case["kind"] == "product":
        batch, rows, cols = case["batch"], case["rows"], case["cols"]
        w = sb.mx(*state["w"], cols)
        x = state["x"]
        if case["x"] == 4:
            x = sb.mx(new(batch, cols // 2, dtype=torch.uint8), new(batch, sb.mx_scale_pitch(cols), dtype=torch.uint8), cols)
            ctx.mx_quantize(state["x"], x)
        y = new(batch, sb.mx_out_pitch(rows), dtype=_type(case["out"]))[:, :rows]
        ctx.mx_gemm(w, x, y, _workspace(ctx.mx_gemm_ws_bytes(w, batch, case["x"] == 4, case["gated"])), gated=case["gated"])
        return y
    router = _router_of(sb, case)
    tokens, k = case["tokens"], case["top_k"]
    if case["kind"] == "route" and case["backward"]:
        d_logits = new(tokens, case["experts"], dtype=torch.float32)
        ctx.route_backward(router, state["logits"], state["ids"], state["d_weights"], d_logits)
        return d_logits
    ids, weights = new(tokens, k, dtype=torch.int32), new(tokens, k, dtype=torch.float32)
    if case["kind"] == "route":
        ctx.route(router, state["logits"], state["bias"], ids, weights)
        return {"ids": ids, "weights": weights}
    up, down = sb.mx(*state["up"], case["hidden"]), sb.mx(*state["down"], case["inner"])
    out = new(tokens, case["hidden"], dtype=torch.bfloat16)
    ws = _workspace(ctx.expert_layer_ws_bytes(router, tokens, up, down, case["x"] == 4))
    ctx.expert_layer(router, state["logits"], state["bias"], state["x"], up, down, out, ids, weights, ws, four_bit=case["x"] == 4)
    return {"out": out, "ids": ids, "weights": weights}


def run(state):
    return _own(state) if own else _plain(state)


# ---- what a pass cannot do without -----------------------------------------------------------------
def _form_bytes(rows, cols):
    return rows * (cols // 2 + cols // 32)


def work(case):
    if case["kind"] == "quantise":
        n = case["rows"] * case["cols"]
        return {"bytes": n * (4 if case["type"] == "fp32" else 2) + n * 2 + n // 32, "flops": 0}
    if case["kind"] == "product":
        rows = case["rows"] * (2 if case["gated"] else 1)
        y = case["batch"] * case["rows"] * (4 if case["out"] == "fp32" else 2)
        return {"bytes": _form_bytes(rows, case["cols"]) + case["batch"] * case["cols"] * 2 + y, "flops": 2 * case["batch"] * rows * case["cols"]}
    tokens, experts, k = case["tokens"], case["experts"], case["top_k"]
    logits = tokens * experts * (4 if case["type"] == "fp32" else 2)
    if case["kind"] == "route":
        return {"bytes": logits + (tokens * (k * 8 + experts * 4) if case["backward"] else tokens * k * 8), "flops": 0}
    used = experts * (1 - (1 - k / experts) ** tokens)          # experts that have a token, were all liked alike
    hidden, inner = case["hidden"], case["inner"]
    stored = used * (_form_bytes(2 * inner, hidden) + _form_bytes(hidden, inner))
    return {"bytes": int(stored) + logits + tokens * k * 8 + tokens * hidden * 4, "flops": 6 * tokens * k * hidden * inner}


# ---- from the definitions, in 64 bits --------------------------------------------------------------
def _two_to(power):
    """2 to whole numbers, from the bits of a double: a power function need not be exact."""
    return (power.long() + 1023 << 52).view(torch.float64)


def _exact_form(x):
    """Values after rounding to the 4-bit form, and the powers of two."""
    x = x.double().reshape(*x.shape[:-1], -1, 32)
    largest = x.abs().max(-1, keepdim=True).values
    power = torch.clamp((largest.view(torch.int64) >> 52) - 1023 - 2, min=-125)
    size = (x.abs() * _two_to(-power)).clamp(max=6.0)
    step = _two_to((size >= 2.0).long() + (size >= 4.0) - 1)
    q = torch.minimum(torch.round(size / step) * step, torch.tensor(6.0, device=x.device, dtype=torch.float64))
    return (torch.sign(x) * q * _two_to(power)).flatten(-2), _two_to(power)[..., 0]


def _exact_stored(w, cols, first, rows):
    codes, scales = w[0][first:first + rows].long(), w[1][first:first + rows, :cols // 32]
    both = torch.empty(rows, cols, dtype=torch.int64, device=codes.device)
    both[:, 0::2], both[:, 1::2] = codes % 16, codes // 16
    size, sign = both % 8, 1 - 2 * (both // 8)
    size = torch.where(size < 2, size * 0.5, (1 + (size % 2) * 0.5) * _two_to(size // 2 - 1))
    return sign * size * _two_to(scales.long() - 127).repeat_interleave(32, 1)


def _exact_scores(case, logits):
    logits = logits.double()
    logits = torch.where(logits.abs() < math.inf, logits, -math.inf)
    if case["score"] == "softmax":
        return logits, torch.nan_to_num(torch.softmax(logits, -1), nan=0.0)
    return logits, torch.sigmoid(logits)


def _exact_route(case, logits, bias):
    logits, p = _exact_scores(case, logits)
    tokens, experts, k = case["tokens"], case["experts"], case["top_k"]
    score = p if bias is None else p + bias.double()
    key = (logits if bias is None else score).clone()
    key[logits == -math.inf] = -math.inf
    if case["groups"] > 1:
        each = experts // case["groups"]
        inside = torch.where(logits == -math.inf, -math.inf, score).reshape(tokens, case["groups"], each)
        first = inside.max(-1)
        second = inside.clone().scatter_(-1, first.indices[..., None], -math.inf).max(-1).values
        left = first.values + torch.where(second == -math.inf, 0.0, second)
        shut = torch.ones_like(left, dtype=torch.bool)
        for _ in range(case["top_groups"]):
            best = (left == left.max(-1, keepdim=True).values).int().argmax(-1, keepdim=True)
            shut.scatter_(1, best, False)
            left.scatter_(1, best, -math.inf)
        key[shut.repeat_interleave(each, 1)] = -math.inf
    ids = torch.full((tokens, k), -1, dtype=torch.int32, device=key.device)
    weights = torch.zeros(tokens, k, dtype=torch.float64, device=key.device)
    for j in range(k):
        top = key.max(-1, keepdim=True).values
        best = (key == top).int().argmax(-1, keepdim=True)
        some = top[:, 0] > -math.inf
        ids[some, j] = best[some, 0].int()
        weights[some, j] = p.gather(1, best)[some, 0]
        key.scatter_(1, best, -math.inf)
    if case["renormalize"]:
        weights = torch.nan_to_num(weights / weights.sum(-1, keepdim=True), nan=0.0)
    return ids, weights


def _exact_route_backward(case, logits, ids, d_weights):
    _, p = _exact_scores(case, logits)
    tokens, experts = p.shape
    taken = torch.zeros(tokens, experts + 1, dtype=torch.float64, device=p.device)
    taken.scatter_(1, torch.where(ids < 0, experts, ids.long()), 1.0)
    taken = taken[:, :experts]
    g = torch.zeros(tokens, experts + 1, dtype=torch.float64, device=p.device)
    g = g.scatter_(1, torch.where(ids < 0, experts, ids.long()), d_weights.double())[:, :experts]
    d_p = g                                                      # of the chosen probabilities
    if case["renormalize"]:
        total = (taken * p).sum(-1, keepdim=True)
        d_p = taken * (g / total - (g * p).sum(-1, keepdim=True) / total ** 2)
        d_p = torch.nan_to_num(d_p, nan=0.0)
    if case["score"] == "sigmoid":
        return d_p * p * (1 - p)
    return p * d_p - p * (p * d_p).sum(-1, keepdim=True)


def _exact_layer(case, state):
    experts, hidden, inner, k = case["experts"], case["hidden"], case["inner"], case["top_k"]
    ids, weights = _exact_route(case, state["logits"], state["bias"])
    x = state["x"].double()
    if case["x"] == 4:
        x, _ = _exact_form(x)
    out = torch.zeros(case["tokens"], hidden, dtype=torch.float64, device=x.device)
    for e in range(experts):
        token, j = torch.nonzero(ids == e, as_tuple=True)
        if len(token) == 0:
            continue
        y = x[token] @ _exact_stored(state["up"], hidden, e * 2 * inner, 2 * inner).T
        h = (y[:, :inner] * torch.sigmoid(y[:, :inner]) * y[:, inner:]).float().to(torch.bfloat16).double()
        if case["x"] == 4:
            h, _ = _exact_form(h)
        y = h @ _exact_stored(state["down"], inner, e * hidden, hidden).T
        out.index_add_(0, token, y * weights[token, j][:, None])
    return {"out": out, "ids": ids, "weights": weights}


def exact(case, seed):
    state = prepare(case, seed)
    if case["kind"] == "quantise":
        return dict(zip(("values", "scales"), _exact_form(state["x"])))
    if case["kind"] == "product":
        x = state["x"].double()
        if case["x"] == 4:
            x, _ = _exact_form(x)
        w = state["w"]
        y = x @ _exact_stored(w, case["cols"], 0, w[0].shape[0]).T
        return y[:, :case["rows"]] * torch.sigmoid(y[:, :case["rows"]]) * y[:, case["rows"]:] if case["gated"] else y
    if case["kind"] == "experts":
        return _exact_layer(case, state)
    if case["backward"]:
        return _exact_route_backward(case, state["logits"], state["ids"], state["d_weights"])
    return dict(zip(("ids", "weights"), _exact_route(case, state["logits"], state["bias"])))
