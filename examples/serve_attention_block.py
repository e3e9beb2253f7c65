"""An attention block of a quantized model answering several requests at once.

    python examples/serve_attention_block.py

Calibrates a fused q/k/v projection and an output projection (W4, rank-r compensation) on random activations, then
serves three requests with their own low-rank adapters: one step with their prompts, of different lengths, and some steps
of one token each.  A step is what a decoder block does between its norms:

    projection          aser_quantize_act_rtn, aser_compensated_forward
    adapters            aser_adapter_forward, in place on the projection's output
    cache               aser_kv_append: norms of queries and keys, rotation, pages
    attention           aser_paged_attention, under a window with sinks
    output projection   as the first, adapters included
"""
from __future__ import annotations

import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2411_07762_amd as aser  # noqa: E402


class Projection:
    """A calibrated linear layer with the adapters of its requests; all buffers on the GPU."""

    def __init__(self, ctx, W, X, r: int, f: int, A, B, scale):
        self.ctx, self.buf = ctx, aser.LayerBuffers(W.shape[0], W.shape[1], r, f, 4, packed=True)
        aser.calibrate_layer(ctx, W, X, self.buf)
        self.A, self.B, self.scale = A, B, scale

    def __call__(self, x, adapter):
        ctx, b, rows = self.ctx, self.buf, x.shape[0]
        codes = torch.empty(rows, b.n, dtype=torch.int8, device=x.device)
        scales = torch.empty(rows, dtype=torch.float32, device=x.device)
        y = torch.empty(rows, b.m, dtype=torch.float32, device=x.device)
        ctx.check(aser.aser_quantize_act_rtn(ctx, x, b.mdiag, 8, codes, scales))
        ctx.ensure_workspace(max(aser.aser_forward_workspace_bytes(rows, b.n, b.m, b.r), aser.aser_adapter_workspace_bytes(rows, b.n, b.m, self.A.shape[1])))
        ctx.check(aser.aser_compensated_forward(ctx, codes, scales, b.codes, aser.ASER_CODES_INT4_PACKED, b.scales, b.L_A, b.L_B, b.r, True, y))
        ctx.check(aser.aser_adapter_forward(ctx, x, adapter, self.A, self.B, self.scale, y, y))
        return y


class Block:
    def __init__(self, ctx, heads: int, kv_heads: int, head_dim: int, hidden: int, adapters: int, rank: int, pages: int, page_size: int, max_tokens: int, int8: bool,
                 window: int, sinks: int, seed: int = 1):
        g = torch.Generator(device="cuda")
        g.manual_seed(seed)

        def rand(*shape):
            return torch.randn(*shape, generator=g, device="cuda")

        def projection(m, n):
            A = (rand(adapters, rank, n) / n ** 0.5).to(torch.bfloat16)
            B = (0.1 * rand(adapters, m, rank)).to(torch.bfloat16)
            return Projection(ctx, rand(m, n) / n ** 0.5, rand(8 * n, n).to(torch.bfloat16), 16, 4, A, B, torch.ones(adapters, device="cuda"))

        self.ctx, self.heads, self.kv_heads, self.d = ctx, heads, kv_heads, head_dim
        self.window, self.sinks = window, sinks
        self.qkv, self.out = projection((heads + 2 * kv_heads) * head_dim, hidden), projection(hidden, heads * head_dim)
        self.q_norm, self.k_norm = 1 + 0.1 * rand(head_dim), 1 + 0.1 * rand(head_dim)
        angle = torch.arange(max_tokens, device="cuda", dtype=torch.float64)[:, None] * 10000.0 ** (-torch.arange(0, head_dim, 2, device="cuda", dtype=torch.float64) / head_dim)
        self.cos, self.sin = angle.cos().float(), angle.sin().float()
        self.cache = aser.KvCache.empty(pages, kv_heads, page_size, head_dim, int8=int8)

    def step(self, x, batch, adapter):
        """x: the new tokens' hidden states (tokens x hidden); adapter: number of each token's adapter."""
        ctx, h, hk, d = self.ctx, self.heads, self.kv_heads, self.d
        y = self.qkv(x, adapter)
        q, k, v = y[:, :h * d], y[:, h * d:(h + hk) * d], y[:, (h + hk) * d:]
        queries = torch.empty(x.shape[0], h * d, dtype=torch.bfloat16, device=x.device)
        ctx.check(aser.aser_kv_append(ctx, q, k, v, self.cache, batch, queries, rope_cos=self.cos, rope_sin=self.sin, q_norm=self.q_norm, k_norm=self.k_norm))
        attended = torch.empty_like(queries)
        ctx.ensure_workspace(aser.aser_paged_attention_workspace_bytes(self.cache, batch, h))
        ctx.check(aser.aser_paged_attention(ctx, queries, self.cache, batch, attended, scale=d ** -0.5, window=self.window, sinks=self.sinks))
        return self.out(attended, adapter)


class Requests:
    """The requests' pages and lengths, as a server keeps them: the next free page to whoever needs one."""

    def __init__(self, n: int, page_size: int, max_tokens: int):
        self.page_size, self.length, self.free = page_size, [0] * n, 0
        self.table = torch.full((n, -(-max_tokens // page_size)), -1, dtype=torch.int32)

    def batch(self, new):
        """The batch in which request s has new[s] new tokens."""
        start = torch.tensor([0] + new).cumsum(0).to(torch.int32)
        for s, n in enumerate(new):
            while (self.table[s] >= 0).sum() * self.page_size < self.length[s] + n:
                self.table[s, int((self.table[s] >= 0).sum())] = self.free
                self.free += 1
            self.length[s] += n
        return aser.KvBatch(start.cuda(), torch.tensor(self.length, dtype=torch.int32).cuda(), self.table.cuda(), tokens=sum(new), max_new=max(new), max_kv=max(self.length))


def run(prompts=(150, 33, 1), steps: int = 6, heads: int = 8, kv_heads: int = 2, head_dim: int = 64, hidden: int = 512, int8: bool = False, window: int = 64,
        sinks: int = 4, page_size: int = 16, seed: int = 1):
    """Returns the block and, per step, (new tokens of each request, x, adapters, output)."""
    ctx = aser.Context(0)
    most = max(prompts) + steps
    requests = Requests(len(prompts), page_size, most)
    block = Block(ctx, heads, kv_heads, head_dim, hidden, 2, 8, len(prompts) * (-(-most // page_size)), page_size, most, int8, window, sinks, seed)
    g = torch.Generator(device="cuda")
    g.manual_seed(seed + 1)
    own = [s % 3 - 1 for s in range(len(prompts))]               # the first request has no adapter
    log = []
    for new in [list(prompts)] + [[1] * len(prompts)] * steps:
        x = torch.randn(sum(new), hidden, generator=g, device="cuda").to(torch.bfloat16)
        adapter = torch.tensor([a for a, n in zip(own, new) for _ in range(n)], dtype=torch.int32, device="cuda")
        log.append((new, x, adapter, block.step(x, requests.batch(new), adapter)))
    torch.cuda.synchronize()
    return block, log


if __name__ == "__main__":
    for new, x, _, y in run()[1]:
        print("%3d new tokens %-16s -> output %s, rms %.3f" % (sum(new), new, tuple(y.shape), y.square().mean().sqrt().item()))
