"""Routing to experts, its gradient and a layer of experts on the GPU, against 64 bits."""
import math

import pytest
import torch

import mx_plain as mp
from mx_shapes import LARGE_LAYERS, LAYERS
from paper_2602_17698_amd import binding as sb

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    c = sb.Context(0, torch.cuda.current_stream().cuda_stream)
    yield c
    c.close()


def gen(seed):
    return torch.Generator().manual_seed(seed)


def make_logits(tokens, experts, kind, seed, masks=True):
    g = gen(seed)
    x = 1.5 * torch.randn(tokens, experts, generator=g)
    if masks:
        x.masked_fill_(torch.rand(tokens, experts, generator=g) < 0.05, -math.inf)
        if tokens > 4:
            x[1] = -math.inf                                     # padding
            x[2, 1:] = -math.inf                                 # one expert left
            x[3] = 0.5                                           # all the same: the lowest indices
            x[4, ::2], x[4, 1::2] = 0.0, -0.0                    # zeros of both signs are the same
            if experts > 4:
                x[0, 3], x[0, 4] = math.nan, math.inf            # not there either
    return x.to(kind)


ROUTERS = [dict(experts=1, top_k=1), dict(experts=8, top_k=2), dict(experts=24, top_k=4, groups=8, top_groups=4), dict(experts=64, top_k=8),
           dict(experts=64, top_k=8, renormalize=False), dict(experts=72, top_k=6, groups=8, top_groups=3), dict(experts=128, top_k=32),
           dict(experts=160, top_k=6, groups=8, top_groups=3, group_score=1, scoring=1), dict(experts=256, top_k=8, groups=8, top_groups=4, scoring=1),
           dict(experts=256, top_k=1, groups=64, top_groups=1), dict(experts=300, top_k=7, scoring=1, renormalize=False),
           dict(experts=512, top_k=16, groups=2, top_groups=1), dict(experts=128, top_k=8, groups=16, top_groups=16, group_score=1)]


@pytest.mark.parametrize("router", ROUTERS, ids=lambda r: "-".join("%s%d" % i for i in r.items()))
@pytest.mark.parametrize("kind", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("biased", [False, True])
@pytest.mark.parametrize("tokens", [1, 29])
def test_route(ctx, router, kind, biased, tokens):
    r = sb.Router(**router)
    wide = make_logits(tokens, r.experts + 3, kind, r.experts + tokens)
    logits = wide[:, :r.experts]
    bias = 0.05 * torch.randn(r.experts, generator=gen(3)) if biased else None
    if biased and r.experts > 8:
        bias[5], bias[6] = math.nan, math.inf
    ids = torch.full((tokens, r.top_k), 77, dtype=torch.int32, device="cuda")
    weights = torch.full((tokens, r.top_k), 7.0, device="cuda")
    ctx.route(r, wide.cuda()[:, :r.experts], bias.cuda() if biased else None, ids, weights)
    want, w = mp.route(r, logits, bias)
    assert torch.equal(ids.cpu(), want)
    # in 64 bits or in fp32 with exp, a sum of up to 512 by 14 additions in a row, two quotients, and an argument that is rounded
    # (2^-24 of at most 20): below 64 roundings
    assert bool(((weights.cpu().double() - w).abs() <= 64 * 2.0 ** -24 * w).all())


@pytest.mark.parametrize("router", ROUTERS, ids=lambda r: "-".join("%s%d" % i for i in r.items()))
@pytest.mark.parametrize("kind,biased", [(torch.float32, True), (torch.bfloat16, False)])
def test_route_of_many_tokens(ctx, router, kind, biased):
    """More tokens than waves have room for one by one; pairs of which one alone leaves the choice open, and an odd last one."""
    test_route(ctx, router, kind, biased, 16 * torch.cuda.get_device_properties(0).multi_processor_count + 1)


@pytest.mark.parametrize("router", [dict(experts=32, top_k=4, groups=4, top_groups=2, scoring=1), dict(experts=256, top_k=8, groups=8, top_groups=4, scoring=1),
                                    dict(experts=96, top_k=6, scoring=1), dict(experts=128, top_k=8, groups=4, top_groups=2, group_score=1),
                                    dict(experts=64, top_k=8)], ids=lambda r: "-".join("%s%d" % i for i in r.items()))
@pytest.mark.parametrize("apart,bias_apart,tokens", [(a, b, 301) for a in (1e-7, 1e-6, 1e-5, 1e-4) for b in (0.0, 1e-6, 0.05)] + [(1e-5, 1e-6, 4301), (1e-5, 0.05, 4301)])
def test_route_of_scores_close_to_each_other(ctx, router, apart, bias_apart, tokens):
    """Scores about as far apart as fp32 can tell: eight logits, repeated with small changes; the choice is that of 64 bits."""
    r, g = sb.Router(**router), gen(tokens)
    logits = torch.randn(tokens, 8, generator=g).repeat(1, r.experts // 8)
    logits += apart * torch.randn(tokens, r.experts, generator=g)
    bias = bias_apart * torch.randn(r.experts, generator=g) if bias_apart else None
    ids = torch.empty(tokens, r.top_k, dtype=torch.int32, device="cuda")
    weights = torch.empty(tokens, r.top_k, device="cuda")
    ctx.route(r, logits.cuda(), bias.cuda() if bias_apart else None, ids, weights)
    want, w = mp.route(r, logits, bias)
    assert torch.equal(ids.cpu(), want)
    assert bool(((weights.cpu().double() - w).abs() <= 64 * 2.0 ** -24 * w).all())


@pytest.mark.parametrize("router", ROUTERS, ids=lambda r: "-".join("%s%d" % i for i in r.items()))
@pytest.mark.parametrize("kind", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("tokens", [1, 29])
def test_route_backward(ctx, router, kind, tokens):
    r = sb.Router(**router)
    logits = make_logits(tokens, r.experts, kind, r.experts, masks=True)
    ids, _ = mp.route(r, logits, None)
    if tokens > 8:
        ids[7, -1] = -1                                          # a choice that was dropped
        ids[8, 0] = r.experts + 1000                             # outside: skipped
    d = torch.randn(tokens, r.top_k, generator=gen(5))
    out = torch.full((tokens, r.experts + 5), 7.0, device="cuda")
    ctx.route_backward(r, logits.cuda(), ids.cuda(), d.cuda(), out[:, :r.experts])
    assert bool((out[:, r.experts:] == 7.0).all())
    got = out[:, :r.experts].cpu().double()
    if tokens > 8:
        ids[8, 0] = -1
    x = torch.where(torch.isfinite(logits.double()), logits.double(), -math.inf).requires_grad_()
    w = mp.chosen_weights(r, x, ids)
    (w * d.double()).sum().backward()
    want = torch.nan_to_num(x.grad)
    want[~torch.isfinite(logits.double())] = 0.0
    # the formula is a weight or p times a difference of d and a sum of d times weights: 64 roundings of these terms (see test_route), and for the
    # difference as many of the sum of magnitudes
    p = mp.chosen_weights(sb.Router(r.experts, r.experts, r.scoring, renormalize=False), x.detach(), torch.arange(r.experts).expand(tokens, -1))
    some = (ids >= 0)
    dd = torch.where(some, d.double().abs(), 0.0)
    scale = torch.zeros_like(p).scatter_add_(1, ids.clamp(min=0).long(), torch.where(some, w.detach(), 0.0)) if r.renormalize else p
    size = torch.zeros_like(p).scatter_add_(1, ids.clamp(min=0).long(), dd) + (dd * w.detach()).sum(-1, keepdim=True)
    assert bool(((got - want).abs() <= 128 * 2.0 ** -24 * scale * size + 1e-37).all()), float(((got - want).abs() / (scale * size + 1e-30)).max())


@pytest.mark.parametrize("scoring", [0, 1])
@pytest.mark.parametrize("renormalize", [False, True])
def test_route_backward_against_differences(ctx, scoring, renormalize):
    """The gradient along random directions against differences of the weights that the formula gives, in 64 bits."""
    r = sb.Router(experts=24, top_k=4, scoring=scoring, renormalize=renormalize)
    logits = make_logits(6, 24, torch.float32, 11, masks=False)
    ids, _ = mp.route(r, logits, None)
    d = torch.randn(6, 4, generator=gen(12))
    out = torch.empty(6, 24, device="cuda")
    ctx.route_backward(r, logits.cuda(), ids.cuda(), d.cuda(), out)
    step = 1e-4
    for seed in range(4):
        v = torch.randn(6, 24, generator=gen(seed)).double()
        ends = [(mp.chosen_weights(r, logits.double() + s * step * v, ids) * d.double()).sum() for s in (1, -1)]
        slope = (ends[0] - ends[1]) / (2 * step)
        # the difference is off by about step^2 times a third derivative (of order |v|^3 |d|, 1e3), the gradient by fp32's roundings
        assert abs(float(slope - (out.cpu().double() * v).sum())) <= 1e-4


# ---- layers ----------------------------------------------------------------------------------------
def make_layer(experts, hidden, inner, seed, extra=0):
    g = gen(seed)
    up, down = mp.random_matrix(experts * 2 * inner, hidden, g, 1), mp.random_matrix(experts * hidden, inner, g, 1)
    descs = [sb.mx(*mp.stored(*m, "cuda", extra)) for m in (up, down)]
    return descs, mp.values(*up).view(experts, 2 * inner, hidden), mp.values(*down).view(experts, hidden, inner)


def check_layer(ctx, tokens, experts, top_k, hidden, inner, four, biased, where):
    r = sb.Router(experts=experts, top_k=top_k, scoring=1 if biased else 0, renormalize=not biased)
    (up, down), up64, down64 = make_layer(experts, hidden, inner, tokens, extra=1 if biased else 0)
    logits = make_logits(tokens, experts, torch.float32, tokens)
    if tokens == 150:
        logits[:, 1:] -= 50.0                                    # nearly all rows to one expert
    bias = 0.05 * torch.randn(experts, generator=gen(3)) if biased else None
    x = (0.05 * torch.randn(tokens, hidden, generator=gen(4))).to(torch.bfloat16)
    out = torch.full((tokens, hidden + 8), 7.0, dtype=torch.bfloat16, device="cuda")
    ids = torch.empty(tokens, top_k, dtype=torch.int32, device="cuda")
    weights = torch.empty(tokens, top_k, device="cuda")
    ws = torch.full((ctx.expert_layer_ws_bytes(r, tokens, up, down, four),), 0xff, dtype=torch.uint8, device="cuda")
    print("[case]", tokens, experts, top_k, hidden, inner, four, biased, flush=True)
    args = (r, logits.cuda(), bias.cuda() if biased else None, x.cuda(), up, down)
    ctx.expert_layer(*args, out[:, :hidden], ids, weights, ws, four_bit=four)
    want_ids, want_w, want, off = mp.layer(r, logits, bias, x.to(where), up64.to(where), down64.to(where), four)
    assert torch.equal(ids.cpu(), want_ids)
    assert bool(((weights.cpu().double() - want_w).abs() <= 64 * 2.0 ** -24 * want_w).all())
    got = out[:, :hidden].to(where).double()
    assert bool(((got - want).abs() <= off).all()), float(((got - want).abs() / off.clamp(min=1e-30)).max())
    assert bool((out[:, hidden:] == 7.0).all())
    first = out.clone()
    ctx.expert_layer(*args, out[:, :hidden], ids, weights, ws, four_bit=four)
    assert torch.equal(first, out)


@pytest.mark.parametrize("tokens,experts,top_k,hidden,inner", LAYERS)
@pytest.mark.parametrize("four", [False, True])
@pytest.mark.parametrize("biased", [False, True])
def test_layer(ctx, tokens, experts, top_k, hidden, inner, four, biased):
    check_layer(ctx, tokens, experts, top_k, hidden, inner, four, biased, "cpu")


@pytest.mark.parametrize("tokens,experts,top_k,hidden,inner", [k[:5] for k in LARGE_LAYERS])
@pytest.mark.parametrize("four", [False, True])
def test_layer_by_large_tiles(ctx, tokens, experts, top_k, hidden, inner, four):
    check_layer(ctx, tokens, experts, top_k, hidden, inner, four, tokens % 400 != 0, "cuda")


def test_layer_without_any_choice(ctx):
    r = sb.Router(experts=4, top_k=2)
    (up, down), _, _ = make_layer(4, 64, 32, 0)
    out = torch.full((9, 64), 7.0, dtype=torch.bfloat16, device="cuda")
    ids, weights = torch.empty(9, 2, dtype=torch.int32, device="cuda"), torch.empty(9, 2, device="cuda")
    ws = torch.full((ctx.expert_layer_ws_bytes(r, 9, up, down),), 0xff, dtype=torch.uint8, device="cuda")
    ctx.expert_layer(r, torch.full((9, 4), -math.inf, device="cuda"), None, torch.ones(9, 64, dtype=torch.bfloat16, device="cuda"), up, down, out, ids,
                     weights, ws)
    assert bool((out == 0).all()) and bool((ids == -1).all()) and bool((weights == 0).all())


@pytest.mark.parametrize("four", [False, True])
def test_layer_in_a_graph(ctx, four):
    """Captured on another stream, replayed with other inputs and eager calls in between."""
    side = torch.cuda.Stream()
    own = sb.Context(0, side.cuda_stream)
    r = sb.Router(experts=8, top_k=2)
    (up, down), _, _ = make_layer(8, 256, 128, 0)
    tokens = 40
    logits, x = torch.empty(tokens, 8, device="cuda"), torch.empty(tokens, 256, dtype=torch.bfloat16, device="cuda")
    out, ids, weights = torch.empty_like(x), torch.empty(tokens, 2, dtype=torch.int32, device="cuda"), torch.empty(tokens, 2, device="cuda")
    ws = torch.empty(own.expert_layer_ws_bytes(r, tokens, up, down, four), dtype=torch.uint8, device="cuda")
    def fill(seed):
        logits.copy_(make_logits(tokens, 8, torch.float32, seed))
        x.copy_(torch.randn(tokens, 256, generator=gen(seed)).to(torch.bfloat16))
        torch.cuda.synchronize()
    def call():
        own.expert_layer(r, logits, None, x, up, down, out, ids, weights, ws, four_bit=four)
    fill(0)
    with torch.cuda.stream(side):
        call()
        side.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            call()
    for turn in range(4):
        fill(turn)
        graph.replay()
        torch.cuda.synchronize()
        kept = out.clone(), ids.clone(), weights.clone()
        out.zero_(), ids.zero_(), weights.zero_()
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            call()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(kept, (out, ids, weights))), turn
    own.close()


@pytest.mark.parametrize("four", [False, True])
def test_the_example_quantises_runs_and_balances(capsys, four):
    import json
    from paper_2602_17698_amd import experts
    assert experts.main(["--hidden", "512", "--inner", "256", "--experts", "16", "--top-k", "4", "--tokens", "512", "--json"] + ["--four-bit"] * four) == 0
    lines = [json.loads(line) for line in capsys.readouterr().out.splitlines()]
    # 4-bit weights of normal distributions are off by some 11 % each, activations as much
    assert [line["stage"] for line in lines] == ["prompt", "16 tokens", "one token", "balance", "balance"]
    assert all(0.02 < line["error"] < 0.5 for line in lines[:3])
    assert lines[4]["variation"] < 0.7 * lines[3]["variation"]
