"""Routing where probabilities are beyond what 32 bits hold: shares of small ones, their gradient, against 64 bits."""
import math

import pytest
import torch

import mx_plain as mp
from paper_2602_17698_amd import binding as sb

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    c = sb.Context(0, torch.cuda.current_stream().cuda_stream)
    yield c
    c.close()


def gen(seed):
    return torch.Generator().manual_seed(seed)


def low_logits(tokens, experts, kind, seed):
    """Tokens whose logits are all, or but for some, far below 0 or far apart."""
    g = gen(seed)
    x = 1.5 * torch.randn(tokens, experts, generator=g)
    level = torch.tensor([0.0, -60.0, -84.0, -87.0, -90.0, -100.0, -104.0, -200.0, -3000.0, -1e30])
    x += level[torch.arange(tokens) % 10][:, None]
    x[torch.arange(tokens) % 3 == 1] *= 1 + 12 * torch.rand(experts, generator=g)      # far apart
    if experts > 4:
        x[::7, 2] = 4.0                                                                 # one far above the rest
        x[5::9, 1] = -math.inf
    x = x.to(kind)
    return torch.where(torch.isfinite(x) | (x == -math.inf), x, torch.finfo(kind).min)


def exact_weights(r, logits, ids):
    """The weights of these choices in 64 bits; shares without the probabilities, which may be below what 64 bits hold."""
    x, some = logits.double().gather(1, ids.clamp(min=0).long()), ids >= 0
    x = torch.where(some, x, -math.inf)
    if r.scoring == 0:
        fine = torch.where(torch.isfinite(logits.double()), logits.double(), -math.inf)
        top = fine.amax(-1, keepdim=True)                                        # (taken away first: beside -1e30 the sum's logarithm is nothing)
        log_p = x - top - torch.log(torch.exp(fine - top).sum(-1, keepdim=True))
    else:
        log_p = torch.where(some, -torch.nn.functional.softplus(-x.clamp(min=-700)) + (x - x.clamp(min=-700)), -math.inf)
    if r.renormalize:
        top = log_p.amax(-1, keepdim=True)
        log_p = log_p - torch.where(top > -math.inf, top, 0.0)
        e = torch.exp(log_p)
        return torch.where(some, e / e.sum(-1, keepdim=True).clamp(min=1e-300), 0.0)
    return torch.where(some, torch.exp(log_p), 0.0)


def check_weights(r, logits, ids, weights):
    want = exact_weights(r, logits, ids)
    # as in the tests of routing: 64 roundings; arguments (differences of logits) are rounded, 2^-24 of up to 88 in weight and sum each: 176 more.  Below the least normal
    # number a weight may be 0
    assert bool(((weights.double() - want).abs() <= 240 * 2.0 ** -24 * want + 2.0 ** -126).all()), float((weights.double() - want).abs().max())
    if r.renormalize:
        some = (ids >= 0).any(-1)
        assert bool(((weights.double().sum(-1) - 1).abs()[some] <= 64 * 2.0 ** -24).all())


ROUTERS = [dict(experts=8, top_k=2), dict(experts=24, top_k=4, groups=8, top_groups=4), dict(experts=64, top_k=8), dict(experts=128, top_k=32),
           dict(experts=256, top_k=8, groups=8, top_groups=4), dict(experts=300, top_k=7)]


@pytest.mark.parametrize("router", ROUTERS, ids=lambda r: "-".join("%s%d" % i for i in r.items()))
@pytest.mark.parametrize("scoring", [0, 1])
@pytest.mark.parametrize("renormalize", [False, True])
@pytest.mark.parametrize("kind", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("tokens", [1, 61, 4301])
def test_weights_of_low_logits(ctx, router, scoring, renormalize, kind, tokens):
    """Without a bias: sigmoids of logits that are all far below 0; groups that leave only experts far below the best."""
    r = sb.Router(scoring=scoring, renormalize=renormalize, **router)
    logits = low_logits(tokens + 4, r.experts, kind, tokens)[4:]                 # (a single token: the one of -90)
    ids, weights = torch.empty(tokens, r.top_k, dtype=torch.int32, device="cuda"), torch.empty(tokens, r.top_k, device="cuda")
    ctx.route(r, logits.cuda(), None, ids, weights)
    if r.groups == 1:                                                            # (groups of which all probabilities are 0 in 64 bits are a matter of the index)
        some = min(tokens, 61)
        assert torch.equal(ids[:some].cpu(), mp.route(r, logits[:some], None)[0])
    check_weights(r, logits, ids.cpu(), weights.cpu())


@pytest.mark.parametrize("router", ROUTERS, ids=lambda r: "-".join("%s%d" % i for i in r.items()))
@pytest.mark.parametrize("scoring", [0, 1])
@pytest.mark.parametrize("renormalize", [False, True])
@pytest.mark.parametrize("tokens", [1, 61, 4301])
def test_weights_of_experts_that_a_bias_prefers(ctx, router, scoring, renormalize, tokens):
    """A bias for the experts with the lowest logits, 30 to 200 below the best."""
    r, g = sb.Router(scoring=scoring, renormalize=renormalize, **router), gen(tokens + 1)
    logits = torch.randn(tokens, r.experts, generator=g)
    low = torch.arange(r.experts) % 2 == 0
    logits[:, low] -= torch.tensor([30.0, 80.0, 87.0, 100.0, 200.0])[torch.arange(tokens) % 5 - 2][:, None]
    bias = torch.where(low, 2.0, 0.0) + 0.01 * torch.randn(r.experts, generator=g)
    ids, weights = torch.empty(tokens, r.top_k, dtype=torch.int32, device="cuda"), torch.empty(tokens, r.top_k, device="cuda")
    ctx.route(r, logits.cuda(), bias.cuda(), ids, weights)
    some = min(tokens, 61)
    assert torch.equal(ids[:some].cpu(), mp.route(r, logits[:some], bias)[0])
    check_weights(r, logits, ids.cpu(), weights.cpu())


@pytest.mark.parametrize("scoring", [0, 1])
@pytest.mark.parametrize("four", [False, True])
def test_layer_of_tokens_with_low_logits(ctx, scoring, four):
    """Tokens whose choices are all far below 0 (by a bias, with softmax) are not zeros."""
    r, tokens, hidden, inner, g = sb.Router(experts=8, top_k=2, scoring=scoring), 5, 64, 32, gen(3)
    up, down = mp.random_matrix(8 * 2 * inner, hidden, g, 1), mp.random_matrix(8 * hidden, inner, g, 1)
    logits = torch.randn(tokens, 8, generator=g)
    logits[:, ::2] -= 95.0
    bias = torch.where(torch.arange(8) % 2 == 0, 2.0, 0.0)
    x = (0.05 * torch.randn(tokens, hidden, generator=g)).to(torch.bfloat16)
    ids, weights = torch.empty(tokens, 2, dtype=torch.int32, device="cuda"), torch.empty(tokens, 2, device="cuda")
    out = torch.empty(tokens, hidden, dtype=torch.bfloat16, device="cuda")
    u, d = (sb.mx(*mp.stored(*m, "cuda")) for m in (up, down))
    ws = torch.empty(ctx.expert_layer_ws_bytes(r, tokens, u, d, four), dtype=torch.uint8, device="cuda")
    ctx.expert_layer(r, logits.cuda(), bias.cuda(), x.cuda(), u, d, out, ids, weights, ws, four_bit=four)
    check_weights(r, logits, ids.cpu(), weights.cpu())
    want_ids, _, want, off = mp.layer(r, logits, bias, x, mp.values(*up).view(8, 2 * inner, hidden), mp.values(*down).view(8, hidden, inner), four)
    assert torch.equal(ids.cpu(), want_ids)
    assert bool(((out.cpu().double() - want).abs() <= off).all())


# ---- the gradient ----------------------------------------------------------------------------------
def check_gradient(ctx, r, logits, ids, d, roundings=128):
    """Against the formulas in 64 bits, each with the magnitudes of its terms: s (|d| + sum |d| s), with sigmoids (1 - p) of that, p (1 - p) |d| without shares."""
    tokens = logits.shape[0]
    out = torch.empty(tokens, r.experts, device="cuda")
    ctx.route_backward(r, logits.cuda(), ids.cuda(), d.cuda(), out)
    some = ids >= 0
    at = ids.clamp(min=0).long()
    x = torch.where(some, logits.double().gather(1, at), -math.inf)
    w, d64 = exact_weights(r, logits, ids), torch.where(some, d.double(), 0.0)
    rest = torch.sigmoid(-x) if r.scoring == 1 else torch.ones_like(x)                 # 1 - p, of its own accuracy
    if r.renormalize:
        g = w * rest * (d64 - (d64 * w).sum(-1, keepdim=True))
        size = w * rest * (d64.abs() + (d64.abs() * w).sum(-1, keepdim=True))
    else:
        assert r.scoring == 1
        g = size = w * rest * d64
    want, sizes = (torch.zeros(tokens, r.experts, dtype=torch.float64).scatter_add_(1, at, torch.where(some, v, 0.0)) for v in (g, size.abs()))
    # below the least normal number a share, p or 1 - p may be 0
    off = roundings * 2.0 ** -24 * sizes + 2.0 ** -126 * (1 + d64.abs().amax())
    got = out.cpu().double()
    assert bool(((got - want).abs() <= off).all()), float(((got - want).abs() / off).max())


@pytest.mark.parametrize("renormalize", [False, True])
@pytest.mark.parametrize("kind", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("experts,top_k,tokens", [(8, 2, 1), (8, 2, 37), (100, 8, 37), (300, 6, 37)])
def test_gradient_of_confident_sigmoids(ctx, renormalize, kind, experts, top_k, tokens):
    """Logits of 3 to 60: the gradient has the factor 1 - p, down to e^-60, as accurate as the rest of it."""
    r, g = sb.Router(experts=experts, top_k=top_k, scoring=1, renormalize=renormalize), gen(tokens)
    logits = (3.0 + 57.0 * torch.rand(tokens, experts, generator=g) ** 2).to(kind)
    ids = torch.stack([torch.randperm(experts, generator=g)[:top_k] for _ in range(tokens)]).int()
    check_gradient(ctx, r, logits, ids, torch.randn(tokens, top_k, generator=g))


@pytest.mark.parametrize("scoring", [0, 1])
@pytest.mark.parametrize("renormalize", [False, True])
def test_gradient_of_choices_whose_logits_are_not_there(ctx, scoring, renormalize):
    """Ids of experts with NaN or infinite logits: their gradient is 0, the others' as if they had not been chosen."""
    r, g = sb.Router(experts=16, top_k=4, scoring=scoring, renormalize=renormalize), gen(2)
    logits, d = torch.randn(4, 16, generator=g), torch.randn(4, 4, generator=g)
    logits[0, 3], logits[1, 3], logits[2, 3] = math.nan, math.inf, -math.inf
    ids = torch.tensor([[1, 3, 5, 7]] * 4, dtype=torch.int32)
    without = ids.clone()
    without[:3, 1] = -1
    out = [torch.empty(4, 16, device="cuda") for _ in range(2)]
    for i, o in zip((ids, without), out):
        ctx.route_backward(r, logits.cuda(), i.cuda(), d.cuda(), o)
    assert bool(torch.isfinite(out[0]).all()) and bool((out[0][:3, 3] == 0).all()) and torch.equal(*out)


@pytest.mark.parametrize("router", ROUTERS, ids=lambda r: "-".join("%s%d" % i for i in r.items()))
@pytest.mark.parametrize("scoring", [0, 1])
@pytest.mark.parametrize("kind", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("tokens", [1, 61])
def test_gradient_of_low_shares(ctx, router, scoring, kind, tokens):
    """Shares among choices that are all far below 0, or below the best: as large as any."""
    r, g = sb.Router(scoring=scoring, **router), gen(tokens + 2)
    logits = low_logits(tokens + 4, r.experts, kind, tokens)[4:]
    ids = mp.route(r, logits, torch.where(torch.arange(r.experts) % 2 == 0, 2.0, 0.0))[0]      # the best, and those that a bias prefers
    if tokens > 8:
        ids[7, -1] = -1
    # (arguments are rounded as in check_weights, of a share and of those it is compared with)
    check_gradient(ctx, r, logits, ids, torch.randn(tokens, r.top_k, generator=g), 2 * 240)


@pytest.mark.parametrize("router", [dict(experts=32, top_k=4, scoring=1), dict(experts=64, top_k=8, scoring=1), dict(experts=256, top_k=8, scoring=1),
                                    dict(experts=64, top_k=8), dict(experts=96, top_k=6, groups=4, top_groups=2, scoring=1)],
                         ids=lambda r: "-".join("%s%d" % i for i in r.items()))
@pytest.mark.parametrize("level", [-30.0, -60.0, -84.0, -86.0, -87.3, -90.0])
@pytest.mark.parametrize("bias", [0.0, 1e-37])
def test_order_of_low_scores(ctx, router, level, bias):
    """Scores that are small probabilities and little else, of logits a unit or some in the last place apart."""
    r, tokens = sb.Router(**router), 67
    g = gen(int(-level))
    step = 2.0 ** -17 if level < -64 else 2.0 ** -19
    logits = torch.full((tokens, r.experts), level) + step * torch.randint(-20, 21, (tokens, r.experts), generator=g)
    logits[:, 0] = 0.0 if r.scoring == 0 else level                              # (softmax: far below the best)
    b = bias * torch.rand(r.experts, generator=g)
    b[0] = -1.0
    ids, weights = torch.empty(tokens, r.top_k, dtype=torch.int32, device="cuda"), torch.empty(tokens, r.top_k, device="cuda")
    ctx.route(r, logits.cuda(), b.cuda(), ids, weights)
    assert torch.equal(ids.cpu(), mp.route(r, logits, b)[0])
    check_weights(r, logits, ids.cpu(), weights.cpu())


@pytest.mark.parametrize("router", [dict(experts=64, top_k=8, scoring=1), dict(experts=256, top_k=8, scoring=1), dict(experts=64, top_k=8),
                                    dict(experts=3, top_k=3, scoring=1), dict(experts=3, top_k=3), dict(experts=6, top_k=2, groups=3, top_groups=1, scoring=1),
                                    dict(experts=96, top_k=6, groups=4, top_groups=2, scoring=1)], ids=lambda r: "-".join("%s%d" % i for i in r.items()))
@pytest.mark.parametrize("level", [-5.0, -30.0, -60.0, -83.7, -85.0, -86.3])
@pytest.mark.parametrize("apart", [0.0, 2.0 ** -21, 2.0 ** -19, 2.0 ** -17])
def test_order_of_low_scores_that_a_bias_evens_out(ctx, router, level, apart):
    """p + bias the same for all experts, to some units in the last place of either."""
    r, g = sb.Router(**router), gen(int(-level))
    logits = (level + 0.4 * torch.rand(1, r.experts, generator=g)).repeat(401, 1)
    logits[:, 0] = 0.3 if r.scoring == 0 else level
    logits[1:] += 2.0 ** (math.frexp(level)[1] - 24) * torch.randint(-1, 2, (400, r.experts), generator=g)
    p = torch.softmax(logits[0].double(), -1) if r.scoring == 0 else torch.sigmoid(logits[0].double())
    most = p[1:].max()
    b = ((2 * most - p) * (1 + apart * torch.randn(r.experts, generator=g).double())).float()
    b[0] = -1.0
    ids, weights = torch.empty(401, r.top_k, dtype=torch.int32, device="cuda"), torch.empty(401, r.top_k, device="cuda")
    ctx.route(r, logits.cuda(), b.cuda(), ids, weights)
    assert torch.equal(ids.cpu(), mp.route(r, logits, b)[0])
    check_weights(r, logits, ids.cpu(), weights.cpu())
