"""A layer of experts with 4-bit floating point weights, as a program uses it: bf16 weights are quantised once, a prompt goes through the layer, then
single tokens, and the router is trained for balance with the gradient of its weights.

    python -m paper_2602_17698_amd.experts [--hidden 2048] [--inner 1024] [--experts 64] [--top-k 8] [--tokens 2048] [--steps 40] [--four-bit] [--json]

Printed for each stage: its time, and how far the layer is from the same one with the bf16 weights (relative, root mean square over some tokens), or how
far the experts' loads are from even (coefficient of variation).  Runs on one GPU through libscalebits.so; weights and tokens are synthetic (seeded).
"""
from __future__ import annotations

import argparse
import json
import time


def quantised(torch, sb, ctx, w):
    """A bf16 matrix in the microscaled form."""
    rows, cols = w.shape
    q = sb.mx(torch.empty(rows, cols // 2, dtype=torch.uint8, device=w.device),
              torch.empty(rows, sb.mx_scale_pitch(cols), dtype=torch.uint8, device=w.device), cols)
    ctx.mx_quantize(w, q)
    return q


class Layer:
    def __init__(self, torch, sb, ctx, hidden, inner, experts, top_k, four_bit, seed=0):
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.torch, self.ctx, self.hidden, self.inner, self.four_bit = torch, ctx, hidden, inner, four_bit
        self.up = (torch.randn(experts * 2 * inner, hidden, generator=g, device="cuda") * hidden ** -0.5).bfloat16()
        self.down = (torch.randn(experts * hidden, inner, generator=g, device="cuda") * inner ** -0.5).bfloat16()
        self.up_q, self.down_q = quantised(torch, sb, ctx, self.up), quantised(torch, sb, ctx, self.down)
        # a router that likes some experts more than others
        self.gate = torch.randn(experts, hidden, generator=g, device="cuda") * hidden ** -0.5
        self.like = 0.5 * torch.randn(experts, generator=g, device="cuda")
        self.router = sb.Router(experts=experts, top_k=top_k)
        self.ws = torch.empty(0, dtype=torch.uint8, device="cuda")

    def logits(self, x):
        return x.float() @ self.gate.t() + self.like

    def __call__(self, x, logits):
        torch, tokens, k = self.torch, x.shape[0], self.router.top_k
        need = self.ctx.expert_layer_ws_bytes(self.router, tokens, self.up_q, self.down_q, self.four_bit)
        if self.ws.numel() < need:
            self.ws = torch.empty(need, dtype=torch.uint8, device="cuda")
        out = torch.empty_like(x)
        ids = torch.empty(tokens, k, dtype=torch.int32, device="cuda")
        weights = torch.empty(tokens, k, dtype=torch.float32, device="cuda")
        self.ctx.expert_layer(self.router, logits, None, x, self.up_q, self.down_q, out, ids, weights, self.ws, four_bit=self.four_bit)
        return out, ids, weights

    def with_bf16_weights(self, x, ids, weights):
        """The same tokens through the weights before quantisation, a token at a time."""
        torch, i = self.torch, self.inner
        out = torch.zeros(x.shape, dtype=torch.float32, device="cuda")
        up, down = self.up.view(-1, 2 * i, self.hidden), self.down.view(-1, self.hidden, i)
        for t, (e, w) in enumerate(zip(ids.tolist(), weights.tolist())):
            for j in range(len(e)):
                if e[j] >= 0:
                    y = up[e[j]].float() @ x[t].float()
                    out[t] += w[j] * (down[e[j]].float() @ (torch.nn.functional.silu(y[:i]) * y[i:]))
        return out


def main(argv=None) -> int:
    import torch

    from paper_2602_17698_amd import binding as sb

    p = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    for name, value in (("hidden", 2048), ("inner", 1024), ("experts", 64), ("top-k", 8), ("tokens", 2048), ("steps", 40)):
        p.add_argument("--" + name, type=int, default=value)
    p.add_argument("--four-bit", action="store_true", help="activations in 4 bits, too")
    p.add_argument("--json", action="store_true")
    a = p.parse_args(argv)

    def say(**line):
        print(json.dumps(line) if a.json else "  ".join("%s %s" % (k, "%.4g" % v if isinstance(v, float) else v) for k, v in line.items()), flush=True)

    ctx = sb.Context(0, torch.cuda.current_stream().cuda_stream)
    layer = Layer(torch, sb, ctx, a.hidden, a.inner, a.experts, a.top_k, a.four_bit)
    g = torch.Generator(device="cuda").manual_seed(1)

    def timed(x):
        logits = layer.logits(x)
        layer(x, logits)
        torch.cuda.synchronize()
        t0 = time.perf_counter()
        out = layer(x, logits)
        torch.cuda.synchronize()
        return out, (time.perf_counter() - t0) * 1e6

    for stage, tokens in (("prompt", a.tokens), ("16 tokens", 16), ("one token", 1)):
        x = torch.randn(tokens, a.hidden, generator=g, device="cuda").bfloat16()
        (out, ids, weights), us = timed(x)
        some = slice(0, min(tokens, 8))
        want = layer.with_bf16_weights(x[some], ids[some], weights[some])
        say(stage=stage, tokens=tokens, us=us, error=float((out[some].float() - want).norm() / want.norm()))

    # Balance: the loss is the sum over tokens of weight * load of its expert; its gradient with respect to the weights is the load itself.
    x = torch.randn(a.tokens, a.hidden, generator=g, device="cuda").bfloat16()
    ids = torch.empty(a.tokens, a.top_k, dtype=torch.int32, device="cuda")
    weights = torch.empty(a.tokens, a.top_k, dtype=torch.float32, device="cuda")
    d_logits = torch.empty(a.tokens, a.experts, dtype=torch.float32, device="cuda")
    for step in range(a.steps + 1):
        logits = layer.logits(x)
        ctx.route(layer.router, logits, None, ids, weights)
        load = torch.bincount(ids.flatten().long(), minlength=a.experts).float() * a.experts / ids.numel()
        if step in (0, a.steps):
            say(stage="balance", step=step, variation=float(load.std()))
        ctx.route_backward(layer.router, logits, ids, load[ids.long()], d_logits)
        layer.like -= 8.0 / a.tokens * d_logits.sum(0)
        layer.gate -= 8.0 / a.tokens * d_logits.t() @ x.float()
    ctx.close()
    return 0


if __name__ == "__main__":
    raise SystemExit(main())
