"""The example of a layer of experts in microscaled 4 bits, against the same steps from the oracle in 64 bits.

Both sides use the layer's codes, scales and factors, and the oracle rounds what the layer keeps in fewer bits: the gated products (bf16, then 4 bits), the
experts' and the dense MLP's outputs (bf16).  fp32 arithmetic moves a rounding to bf16 by a step now and then, and of the values so moved about one in 2^6 crosses a border of
its 4-bit code, a step of up to a third of it: far below 1 % of the output's norm, beside the last rounding's 2^-9."""
import os
import sys

import numpy as np
import pytest
import torch

from oracle import mx4_oracle as orc

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
import serve_expert_layer as example  # noqa: E402

pytestmark = pytest.mark.gpu


def f64(t):
    return t.detach().double().cpu().numpy()


def bf16(x):
    return torch.from_numpy(np.asarray(x, np.float32)).to(torch.bfloat16).double().numpy()


def quantized(x):
    return orc.values(*orc.quantize(x.astype(np.float32)))[:, :x.shape[1]]


def weight(p, e):
    """The numbers of matrix e."""
    codes, scales = p.w.codes[e].cpu().numpy(), p.w.scales[e].cpu().numpy()
    codes = codes.transpose(0, 3, 1, 2, 4).reshape(codes.shape[0] * 16, -1)[:p.m]
    scales = scales.transpose(0, 2, 1, 3).reshape(scales.shape[0] * 16, -1)[:p.m]
    return orc.values(orc.unpack(codes, np.zeros((1, p.m, 4), np.uint8))[0], scales)[:, :p.n]


def product(p, e, x):
    return orc.product(x, weight(p, e), f64(p.L_A[e]), f64(p.L_B[e]))[0]


@pytest.mark.parametrize("sizes", [dict(), dict(prompt=700, hidden=384, inner=1300, experts=4, top_k=2, groups=1, r=8, steps=1)], ids=["small", "tiles"])
def test_served_layer(sizes):
    layer, log = example.run(**sizes)
    groups = layer.groups
    for x, got, plan, logits in log:
        xv = quantized(f64(x))
        ids, weights = orc.route(f64(logits), layer.top_k, f64(layer.bias), True, groups, max(1, groups // 2), 2)
        assert np.array_equal(plan.ids.cpu().numpy(), ids)
        want = bf16(product(layer.dense_down, 0, quantized(bf16(orc.gated(product(layer.dense_up, 0, xv))))))
        for e in range(layer.experts):
            rows, choice = np.nonzero(ids == e)
            if rows.size:
                y = bf16(product(layer.down, e, quantized(bf16(orc.gated(product(layer.up, e, xv[rows]))))))
                want[rows] += weights[rows, choice][:, None] * y
        rel = np.linalg.norm(f64(got) - want) / np.linalg.norm(want)
        assert rel <= 0.01, rel


def test_factors_of_the_example_compensate():
    """The calibrated projections are nearer to their weights' outputs than the codes alone (weights as the example's seed makes them)."""
    layer, _ = example.run(prompt=1, steps=0)
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    hidden, inner = layer.hidden, layer.inner
    for shape in ((8 * hidden, hidden), (8 * inner, inner)):
        torch.randn(*shape, generator=g, device="cuda")
    W = f64(torch.randn(2 * inner, hidden, generator=g, device="cuda") / hidden ** 0.5)
    x = np.random.default_rng(0).standard_normal((400, hidden))
    bare, full = x @ weight(layer.up, 0).T, product(layer.up, 0, x)
    assert np.linalg.norm(full - x @ W.T) < 0.97 * np.linalg.norm(bare - x @ W.T)
