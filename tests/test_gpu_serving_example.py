"""The example of a quantized attention block that serves requests, against the same steps from the oracles in 64 bits.

Both sides use the block's codes, scales and factors, and the oracles round what the block keeps in fewer bits: queries, keys, values (or their
8-bit codes) and the attention's output.  What differs is fp32 arithmetic, which now and then moves one of these roundings by a
step, and a code of the second projection's 8-bit input with it (1 / 127 of a token's largest value): 1 % of the output's norm; 3 % with an
8-bit cache, whose steps are larger.
"""
import os
import sys

import numpy as np
import pytest
import torch

from oracle import aser_oracle as base
from oracle import serving_oracle as orc

from gpu_util import unpack_int4
from test_gpu_parity import say

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
import serve_attention_block as example  # noqa: E402

pytestmark = pytest.mark.gpu


def f64(t):
    return t.detach().float().cpu().numpy().astype(np.float64)


def bf16(x):
    return torch.from_numpy(np.asarray(x, np.float32)).to(torch.bfloat16).float().numpy().astype(np.float64)


def stored(x, int8):
    """Keys or values as the cache holds them."""
    if not int8:
        return bf16(x)
    top = np.abs(x).max(-1, keepdims=True)
    scale = np.where(top == 0, 1.0, top / 127.0)
    return np.rint(x / scale) * scale


def projected(p, x, ids):
    b = p.buf
    y = base.compensated_forward(x.astype(np.float32), f64(b.mdiag).astype(np.float32), unpack_int4(b.codes.cpu().numpy()), f64(b.scales).astype(np.float32),
                                 f64(b.L_A).astype(np.float32), f64(b.L_B).astype(np.float32), 8)
    return orc.adapters(x, ids, f64(p.A), f64(p.B), f64(p.scale), y)[0]


@pytest.mark.parametrize("int8,window,bar", [(False, 64, 0.01), (True, 0, 0.03)], ids=["bf16_window", "int8"])
def test_served_block(int8, window, bar):
    say("served block int8=%s" % int8)
    block, log = example.run(int8=int8, window=window)
    h, hk, d = block.heads, block.kv_heads, block.d
    cos, sin, qn, kn = (t.cpu().numpy() for t in (block.cos, block.sin, block.q_norm, block.k_norm))
    n = len(log[0][0])
    keys, values = [np.zeros((0, hk, d))] * n, [np.zeros((0, hk, d))] * n
    for new, x, adapter, got in log:
        ids = adapter.cpu().numpy()
        y = projected(block.qkv, f64(x), ids).reshape(len(ids), -1, d)
        att = np.zeros((len(ids), h, d))
        at = 0
        for s, c in enumerate(new):
            rows, pos = slice(at, at + c), np.arange(len(keys[s]), len(keys[s]) + c)
            at += c
            q = bf16(orc.turned(y[rows, :h], pos, cos, sin, False, qn, 1e-6))
            keys[s] = np.concatenate([keys[s], stored(orc.turned(y[rows, h:h + hk], pos, cos, sin, False, kn, 1e-6), int8)])
            values[s] = np.concatenate([values[s], stored(y[rows, h + hk:], int8)])
            t = len(keys[s])
            page = 1 << max(4, (t - 1).bit_length())                # one page for the oracle
            k, v = np.zeros((1, hk, page, d)), np.zeros((1, hk, page, d))
            k[0, :, :t], v[0, :, :t] = keys[s].transpose(1, 0, 2), values[s].transpose(1, 0, 2)
            att[rows] = orc.attention(q, k, v, np.zeros((1, 1), int), np.array([0, c]), np.array([t]), d ** -0.5, window, block.sinks)[0]
        want = projected(block.out, bf16(att).reshape(len(ids), -1), ids)
        rel = np.linalg.norm(f64(got) - want) / np.linalg.norm(want)
        say("%s new tokens: relative difference %.2e" % (new, rel))
        assert rel <= bar
