"""Layers of experts for up to 8 tokens, whose choices and lists are one launch, and for a token more; with groups, biases, both scorings and types of logits."""
import math

import pytest
import torch

import mx_plain as mp
from paper_2602_17698_amd import binding as sb

pytestmark = pytest.mark.gpu

# experts, choices, and the registers of a lane that the launch for both needs (None: two launches)
ROUTERS = [(dict(experts=4, top_k=4), 1), (dict(experts=24, top_k=4, groups=8, top_groups=4), 1), (dict(experts=72, top_k=6, groups=8, top_groups=3), 2),
           (dict(experts=128, top_k=32), 2), (dict(experts=160, top_k=6, groups=8, top_groups=3, group_score=1), 4), (dict(experts=256, top_k=8), 4),
           (dict(experts=256, top_k=32, groups=8, top_groups=4), 4), (dict(experts=300, top_k=7), None)]
TOKENS = [1, 2, 5, 8, 9]


@pytest.fixture(scope="module")
def ctx():
    c = sb.Context(0, torch.cuda.current_stream().cuda_stream)
    yield c
    c.close()


@pytest.mark.parametrize("router", [k[0] for k in ROUTERS], ids=lambda r: "-".join("%s%d" % i for i in r.items()))
@pytest.mark.parametrize("tokens", TOKENS)
@pytest.mark.parametrize("scoring,biased,renormalize", [(0, False, True), (0, True, False), (1, True, True)])
@pytest.mark.parametrize("kind,four", [(torch.float32, False), (torch.bfloat16, True)])
def test_layer_of_few_tokens(ctx, router, tokens, scoring, biased, renormalize, kind, four):
    r, hidden, inner = sb.Router(scoring=scoring, renormalize=renormalize, **router), 64, 32
    g = torch.Generator().manual_seed(r.experts + tokens)
    up, down = mp.random_matrix(r.experts * 2 * inner, hidden, g, 1), mp.random_matrix(r.experts * hidden, inner, g, 1)
    logits = 1.5 * torch.randn(tokens, r.experts, generator=g)
    logits.masked_fill_(torch.rand(tokens, r.experts, generator=g) < 0.05, -math.inf)
    if tokens > 1:
        logits[1] = -math.inf                                    # padding
    if tokens > 4:
        logits[2, 3:] = -math.inf                                # fewer experts than choices
        logits[3] = 0.5                                          # all the same: the lowest indices
        logits[4] = logits[0]                                    # the same choices twice
    logits = logits.to(kind)
    bias = 0.05 * torch.randn(r.experts, generator=g) if biased else None
    x = (0.05 * torch.randn(tokens, hidden, generator=g)).to(torch.bfloat16)
    u, d = (sb.mx(*mp.stored(*m, "cuda")) for m in (up, down))
    out = torch.full((tokens, hidden + 8), 7.0, dtype=torch.bfloat16, device="cuda")
    ids, weights = torch.full((tokens, r.top_k), 77, dtype=torch.int32, device="cuda"), torch.full((tokens, r.top_k), 7.0, device="cuda")
    ws = torch.full((ctx.expert_layer_ws_bytes(r, tokens, u, d, four),), 0xff, dtype=torch.uint8, device="cuda")
    print("[case]", r.experts, tokens, scoring, biased, kind, four, flush=True)
    ctx.expert_layer(r, logits.cuda(), bias.cuda() if biased else None, x.cuda(), u, d, out[:, :hidden], ids, weights, ws, four_bit=four)
    want_ids, want_w, want, off = mp.layer(r, logits, bias, x, mp.values(*up).view(r.experts, 2 * inner, hidden),
                                           mp.values(*down).view(r.experts, hidden, inner), four)
    assert torch.equal(ids.cpu(), want_ids)
    assert bool(((weights.cpu().double() - want_w).abs() <= 64 * 2.0 ** -24 * want_w).all())        # (see the tests of routing)
    got = out.cpu().double()
    assert bool(((got[:, :hidden] - want).abs() <= off).all()) and bool((got[:, hidden:] == 7.0).all())
