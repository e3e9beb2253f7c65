"""A layer of experts of a quantized model in microscaled 4 bits, answering prompts and then single tokens.

    python examples/serve_expert_layer.py

Calibrates every expert's two projections, and those of a dense MLP that all tokens go through, on random activations: the statistics,
whitening and reconstruction of a layer, with aser_mx4_quantize as the weight quantizer in front of aser_quant_target.  A step is what the MLP of a
decoder block does between its norms:

    router              aser_route_experts on the logits: sigmoid scores, a bias, groups of experts
    tokens              aser_mx4_quantize, once for all experts
    gate and up         aser_expert_forward, rows by their experts, silu(gate) * up behind the low-rank branch
    down                aser_mx4_quantize, aser_expert_forward
    dense MLP           aser_mx4_forward, gated, and again
    sum                 aser_expert_combine on top of the dense MLP's output
"""
from __future__ import annotations

import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2411_07762_amd as aser  # noqa: E402

BF16 = torch.bfloat16


def calibrated(ctx, W, X, r: int, codes: aser.Mx4):
    """Quantizes W (m x n) into `codes` and returns the factors that make up for the error on inputs like X, in 16 bits."""
    m, n = W.shape
    buf = aser.LayerBuffers(m, n, r, 0, 4, False)
    ctx.ensure_workspace(aser.aser_workspace_bytes(m, n, r))
    ctx.check(aser.aser_gram_accumulate(ctx, X, buf.G, buf.abs_sum, buf.count))
    ctx.check(aser.aser_smooth_outliers(ctx, W, buf.abs_sum, buf.count, 0, buf.idx, buf.mdiag))       # experts share their input: nothing is smoothed
    Wq = torch.empty_like(W)
    ctx.check(aser.aser_mx4_quantize(ctx, W, codes, values=Wq))
    ctx.check(aser.aser_quant_target(ctx, W, buf.mdiag, Wq, buf.T))
    status, _ = aser.aser_whiten(ctx, buf.G, buf.mdiag, 0.01, buf.S)
    ctx.check(status)
    ctx.check(aser.aser_error_reconstruct(ctx, buf.T, buf.S, r, buf.L_A, buf.L_B, buf.sigma)[0])
    return buf.L_A.to(BF16), buf.L_B.to(BF16)


class Projections:
    """Calibrated projections on one input, m x n each, a matrix per expert (or one)."""

    def __init__(self, ctx, weights, X, r: int):
        m, n = weights[0].shape
        self.w = aser.Mx4.empty(m, n, len(weights))
        made = [calibrated(ctx, W, X, r, aser.Mx4(self.w.codes[e], self.w.scales[e], n, m)) for e, W in enumerate(weights)]
        self.L_A, self.L_B = torch.stack([a for a, _ in made]), torch.stack([b for _, b in made])
        self.m, self.n, self.r = m, n, r


class Layer:
    def __init__(self, ctx, hidden: int, inner: int, experts: int, top_k: int, groups: int, r: int, seed: int):
        g = torch.Generator(device="cuda")
        g.manual_seed(seed)

        def rand(*shape):
            return torch.randn(*shape, generator=g, device="cuda")

        def projections(count, m, n, X):
            return Projections(ctx, [rand(m, n) / n ** 0.5 for _ in range(count)], X, r)

        self.ctx, self.hidden, self.inner, self.experts, self.top_k, self.groups = ctx, hidden, inner, experts, top_k, groups
        x, h = rand(8 * hidden, hidden).to(BF16), (rand(8 * inner, inner) * 0.5).to(BF16)
        self.up, self.down = projections(experts, 2 * inner, hidden, x), projections(experts, hidden, inner, h)
        self.dense_up, self.dense_down = projections(1, 2 * inner, hidden, x), projections(1, hidden, inner, h)
        self.router, self.bias = rand(hidden, experts) / hidden ** 0.5, 0.05 * rand(experts)

    def quantized(self, x):
        out = aser.Mx4.empty(*x.shape)
        self.ctx.check(aser.aser_mx4_quantize(self.ctx, x, out))
        return out

    def dense(self, x, p: Projections, rows: int, swiglu: bool):
        y = torch.empty(rows, p.m // 2 if swiglu else p.m, dtype=BF16, device="cuda")
        self.ctx.ensure_workspace(aser.aser_mx4_forward_workspace_bytes(rows, p.n, p.m, p.r))
        w = aser.Mx4(p.w.codes[0], p.w.scales[0], p.n, p.m)
        self.ctx.check(aser.aser_mx4_forward(self.ctx, x, w, y, L_A=p.L_A[0], L_B=p.L_B[0], swiglu=swiglu))
        return y

    def expert(self, x, p: Projections, plan, gather: bool):
        y = torch.zeros(plan.positions, p.m // 2 if gather else p.m, dtype=BF16, device="cuda")        # rows behind the last position stay as they are
        self.ctx.ensure_workspace(aser.aser_expert_forward_workspace_bytes(plan.positions, p.n, p.m, self.experts, p.r))
        self.ctx.check(aser.aser_expert_forward(self.ctx, x, p.w, plan, y, gather=gather, swiglu=gather, L_A=p.L_A, L_B=p.L_B))
        return y

    def step(self, x):
        """x: tokens x hidden, bfloat16; returns the layer's output and the plan of who went where."""
        ctx, rows = self.ctx, x.shape[0]
        logits = x.float() @ self.router
        plan = aser.ExpertPlan.empty(rows, self.top_k, self.experts)
        ctx.ensure_workspace(aser.aser_route_workspace_bytes(rows, self.experts, self.top_k))
        ctx.check(aser.aser_route_experts(ctx, logits, plan, bias=self.bias, sigmoid=True, groups=self.groups, top_groups=max(1, self.groups // 2), group_top=2))
        codes = self.quantized(x)
        out = self.dense(self.quantized(self.dense(codes, self.dense_up, rows, True)), self.dense_down, rows, False)
        made = self.expert(self.quantized(self.expert(codes, self.up, plan, True)), self.down, plan, False)
        ctx.check(aser.aser_expert_combine(ctx, made, plan, out, Y0=out))
        return out, plan, logits


def run(prompt: int = 180, steps: int = 3, batch: int = 5, hidden: int = 256, inner: int = 160, experts: int = 8, top_k: int = 3, groups: int = 4, r: int = 16, seed: int = 1):
    """Returns the layer and, per step, (x, output, plan, logits): a prompt's tokens, then a token of each of `batch` requests at a time."""
    layer = Layer(aser.Context(0), hidden, inner, experts, top_k, groups, r, seed)
    g = torch.Generator(device="cuda")
    g.manual_seed(seed + 1)
    log = []
    for rows in [prompt] + [batch] * steps:
        x = torch.randn(rows, hidden, generator=g, device="cuda").to(BF16)
        log.append((x, *layer.step(x)))
    torch.cuda.synchronize()
    return layer, log


if __name__ == "__main__":
    for x, y, plan, _ in run()[1]:
        print("%3d tokens -> output %s, rms %.3f; rows of each expert %s" % (x.shape[0], tuple(y.shape), y.float().square().mean().sqrt().item(), plan.offsets.diff().tolist()))
