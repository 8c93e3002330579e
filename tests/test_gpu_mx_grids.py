"""More tokens than a launch takes: what lies on both sides of the pieces' border, and at the end, against 64 bits."""
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


@pytest.mark.parametrize("kind", [torch.float32, torch.bfloat16])
def test_routing_of_more_tokens_than_a_launch_takes(ctx, kind):
    border, experts, k = 1 << 25, 8, 2
    tokens, r = border + 77, sb.Router(experts=experts, top_k=k)
    g = torch.Generator(device="cuda").manual_seed(1)
    logits = torch.randn(tokens, experts, device="cuda", generator=g).to(kind)
    ids, weights = torch.full((tokens, k), 77, dtype=torch.int32, device="cuda"), torch.full((tokens, k), 7.0, device="cuda")
    print("[case]", kind, flush=True)
    ctx.route(r, logits, None, ids, weights)
    d, d_logits = torch.randn(tokens, k, device="cuda", generator=g), torch.full((tokens, experts), 7.0, device="cuda")
    ctx.route_backward(r, logits, ids, d, d_logits)
    assert bool(((ids >= 0) & (ids < experts)).all()) and bool((d_logits != 7.0).all())
    for part in (slice(0, 50), slice(border - 50, border + 77)):
        some = logits[part].cpu()
        want, w = mp.route(r, some, None)
        assert torch.equal(ids[part].cpu(), want)
        assert bool(((weights[part].cpu().double() - w).abs() <= 64 * 2.0 ** -24 * w).all())
        x = some.double().requires_grad_()
        (mp.chosen_weights(r, x, want) * d[part].cpu().double()).sum().backward()
        # 128 roundings of a share (below 1) times |d| and the sum of the shares' |d|
        size = 2 * d[part].cpu().double().abs().amax(-1, keepdim=True)
        assert bool(((d_logits[part].cpu().double() - x.grad).abs() <= 128 * 2.0 ** -24 * size).all())


def test_layer_of_more_tokens_than_a_launch_of_the_sum_takes(ctx):
    border, experts, hidden, inner = 1 << 23, 2, 32, 32
    tokens, r = border + 77, sb.Router(experts=experts, top_k=1, renormalize=False)
    g = torch.Generator().manual_seed(2)
    up, down = mp.random_matrix(experts * 2 * inner, hidden, g, 1), mp.random_matrix(experts * hidden, inner, g, 1)
    u, d = (sb.mx(*mp.stored(*m, "cuda")) for m in (up, down))
    g = torch.Generator(device="cuda").manual_seed(3)
    logits = torch.randn(tokens, experts, device="cuda", generator=g)
    x = (0.05 * torch.randn(tokens, hidden, device="cuda", generator=g)).to(torch.bfloat16)
    out = torch.empty(tokens, hidden, dtype=torch.bfloat16, device="cuda")
    ids, weights = torch.empty(tokens, 1, dtype=torch.int32, device="cuda"), torch.empty(tokens, 1, device="cuda")
    ws = torch.empty(ctx.expert_layer_ws_bytes(r, tokens, u, d), dtype=torch.uint8, device="cuda")
    print("[case]", tokens, flush=True)
    ctx.expert_layer(r, logits, None, x, u, d, out, ids, weights, ws)
    for part in (slice(0, 50), slice(border - 50, border + 77)):
        want_ids, _, want, off = mp.layer(r, logits[part].cpu(), None, x[part].cpu(), mp.values(*up).view(experts, 2 * inner, hidden),
                                          mp.values(*down).view(experts, hidden, inner), False)
        assert torch.equal(ids[part].cpu(), want_ids)
        assert bool(((out[part].cpu().double() - want).abs() <= off).all())


@pytest.mark.parametrize("gated", [False, True])
def test_product_with_more_rows_of_w_than_a_launch_takes(ctx, gated):
    border, cols = (32 if gated else 64) << 22, 32
    outs = border + 77
    rows = outs * (2 if gated else 1)
    g = torch.Generator(device="cuda").manual_seed(4)
    codes = torch.randint(0, 256, (rows, cols // 2), dtype=torch.uint8, device="cuda", generator=g)
    scales = torch.randint(118, 124, (rows, 4), dtype=torch.uint8, device="cuda", generator=g)
    x = torch.randn(1, cols, device="cuda", generator=g).to(torch.bfloat16)
    y = torch.full((1, sb.mx_out_pitch(outs)), 7.0, device="cuda")
    print("[case]", rows, flush=True)
    ctx.mx_gemm(sb.mx(codes, scales, cols), x, y[:, :outs], None, gated=gated)
    assert bool((y[:, outs:] == 7.0).all())
    for first, last in ((0, 50), (border - 50, outs)):
        part = torch.cat([torch.arange(first, last) + half * outs for half in range(2 if gated else 1)]).cuda()
        want, off = mp.product(x.cpu().double(), mp.values(mp.unpack(codes[part].cpu()), scales[part, :1].cpu()), gated)
        assert bool(((y[:, first:last].cpu().double() - want).abs() <= off + 2.0 ** -24 * (want.abs() + off)).all())
