"""A layer of experts with 4-bit floating point weights, as a program uses it: bf16 weights are quantised once, a prompt goes through the layer, then
single tokens, and the router is trained for balance with the gradient of its weights.

    python -m paper_2602_17698_amd.experts [--hidden 2048] [--inner 1024] [--experts 64] [--top-k 8] [--tokens 2048] [--steps 40] [--four-bit] [--json]
                                           [--heads 16 --kv-heads 4]

With --heads there is attention ahead of the experts: a prompt's keys, at rotary positions, and values go into a paged cache in 4 bits, and single tokens are
decoded behind it, by a graph that is captured once.

Printed for each stage: its time, and how far the layer is from the same one with the bf16 weights (relative, root mean square over some tokens), or how
far the experts' loads are from even (coefficient of variation); with attention how far its output is from the one with keys and values in 16 bits.  Runs on one GPU through libscalebits.so; weights and tokens are synthetic (seeded).
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


class Attention:
    """Attention of one sequence with 4-bit projections and a 4-bit cache of pages of 64 tokens."""

    def __init__(self, torch, sb, ctx, hidden, heads, kv_heads, most, seed=2):
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.torch, self.sb, self.ctx, self.heads, self.kv_heads, self.dim = torch, sb, ctx, heads, kv_heads, hidden // heads // 32 * 32 or 32
        self.widths = [heads * self.dim, kv_heads * self.dim, kv_heads * self.dim]
        self.project = quantised(torch, sb, ctx, (torch.randn(sum(self.widths), hidden, generator=g, device="cuda") * hidden ** -0.5).bfloat16())
        self.back = quantised(torch, sb, ctx, (torch.randn(hidden, self.widths[0], generator=g, device="cuda") * self.widths[0] ** -0.5).bfloat16())
        pages = (most + 63) // 64
        self.cache = sb.kv_cache(*(torch.zeros(pages, kv_heads, 64, n, dtype=torch.uint8, device="cuda")
                                   for n in (self.dim // 2, sb.mx_scale_pitch(self.dim)) * 2), self.dim)
        self.table = torch.randperm(pages, generator=torch.Generator().manual_seed(seed)).int().cuda().view(1, pages)
        self.length = torch.zeros(1, dtype=torch.int32, device="cuda")
        self.rotary = sb.rotary(torch.tensor(sb.rotary_turns(self.dim, 500000.0), dtype=torch.float64, device="cuda"))

    def buffers(self, tokens):
        """What a pass over so many new tokens writes: projections, turned queries, attention, output; its descriptor and workspace."""
        torch, sb = self.torch, self.sb
        new = lambda n: torch.empty(tokens, n, dtype=torch.bfloat16, device="cuda")  # noqa: E731
        seqs = sb.sequences(torch.tensor([0, tokens], dtype=torch.int32, device="cuda"), self.length, self.table, max_new=tokens)
        need = max(self.ctx.mx_gemm_ws_bytes(self.project, tokens), self.ctx.mx_gemm_ws_bytes(self.back, tokens),
                   self.ctx.kv_attention_ws_bytes(self.cache, seqs, tokens, self.heads))
        return new(sum(self.widths)), new(self.widths[0]), new(self.widths[0]), new(self.back.rows), seqs, torch.empty(max(need, 1), dtype=torch.uint8, device="cuda")

    def __call__(self, x, buffers):
        """x's tokens are the sequence's next; self.length counts them already."""
        qkv, turned, mixed, out, seqs, ws = buffers
        self.ctx.mx_gemm(self.project, x, qkv, ws)
        q, k, v = (t.unflatten(1, (-1, self.dim)) for t in qkv.split(self.widths, 1))
        turned, mixed = turned.view(q.shape), mixed.view(q.shape)
        self.ctx.kv_store(self.cache, seqs, k, v, rotary=self.rotary, q=q, q_out=turned)
        self.ctx.kv_attention(self.cache, seqs, turned, mixed, ws)
        self.ctx.mx_gemm(self.back, mixed.flatten(1), out, ws)
        return out

    def in_16_bits(self, qkv, rows):
        """The mixed values of some rows with the keys and values of a prompt as they were projected."""
        torch = self.torch
        q, k, v = (t.float().unflatten(1, (-1, self.dim)) for t in qkv.split(self.widths, 1))
        at = torch.arange(len(q), dtype=torch.int32, device="cuda")
        for t in (q, k):
            self.ctx.rotate(self.rotary, at, t, t)
        k, v = (t.repeat_interleave(self.heads // self.kv_heads, 1).transpose(0, 1) for t in (k, v))
        scores = q[rows].transpose(0, 1) @ k.transpose(1, 2).contiguous() * self.dim ** -0.5
        scores.masked_fill_(at > at[rows][:, None], float("-inf"))
        return (torch.softmax(scores, -1) @ v.contiguous()).transpose(0, 1).flatten(1)


def main(argv=None) -> int:
    import torch

    from paper_2602_17698_amd import binding as sb

    p = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    for name, value in (("hidden", 2048), ("inner", 1024), ("experts", 64), ("top-k", 8), ("tokens", 2048), ("steps", 40)):
        p.add_argument("--" + name, type=int, default=value)
    p.add_argument("--heads", type=int, default=0, help="attention ahead of the experts, with so many heads of queries")
    p.add_argument("--kv-heads", type=int, default=4)
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

    if a.heads:
        steps = 8
        attention = Attention(torch, sb, ctx, a.hidden, a.heads, a.kv_heads, a.tokens + steps + 1)
        x = torch.randn(a.tokens, a.hidden, generator=g, device="cuda").bfloat16()
        buffers = attention.buffers(a.tokens)
        attention.length.fill_(a.tokens)
        attention(x, buffers)
        torch.cuda.synchronize()
        t0 = time.perf_counter()
        attention(x, buffers)
        torch.cuda.synchronize()
        us = (time.perf_counter() - t0) * 1e6
        rows = slice(max(0, a.tokens - 64), a.tokens)
        want = attention.in_16_bits(buffers[0], rows)
        say(stage="attention, prompt", tokens=a.tokens, us=us, error=float((buffers[2][rows].float() - want).norm() / want.norm()))
        # single tokens: a graph of the whole pass, replayed with the sequence's new length
        side = torch.cuda.Stream()
        own = attention.ctx = sb.Context(0, side.cuda_stream)
        one, buffers = x[:1].clone(), attention.buffers(1)
        attention.length.add_(1)
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            attention(one, buffers)
        side.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            attention(one, buffers)
        torch.cuda.synchronize()
        t0 = time.perf_counter()
        for _ in range(steps):
            attention.length.add_(1)
            graph.replay()
            one.copy_(buffers[3])
        torch.cuda.synchronize()
        say(stage="attention, one token", tokens=1, us=(time.perf_counter() - t0) * 1e6 / steps, length=int(attention.length))
        own.close()

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
