"""Layers in microscaled 4 bits and layers of experts against the float64 oracle.

Tolerances.  Quantization and choices are exact.  A product's sums are held in fp32: an instruction adds 128 exact products to one (four for the rank-r
branch), so a sum of n channels and r ranks passes through at most n / 128 + 1 + r + 16 fp32 additions (16: the parts of wavefronts), each off by
at most 2^-23 of the sum of magnitudes (one ulp, should the instruction truncate), P through n / 8 + 16.  Rounding to the type of the output adds half a step."""
import numpy as np
import pytest
import torch

import paper_2411_07762_amd as aser
from oracle import mx4_oracle as orc

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.fixture(scope="module")
def ctx():
    return aser.Context(0)


def sums_off(n, r):
    return (n / 128 + 17 + r + (n / 8 + 16 if r else 0)) * 2.0 ** -23


def close(got, want, tol):
    got = got.double().cpu().numpy()
    bad = ~(np.abs(got - want) <= tol)
    both = np.isnan(got) & np.isnan(want)
    assert not (bad & ~both).any(), "worst %g of %g allowed" % (np.nanmax(np.abs(got - want)), np.nanmax(tol))


def rounding(want, dtype):
    return np.abs(want) * (2.0 ** -8 if dtype == torch.bfloat16 else 2.0 ** -24)


def dev(a, dtype=None):
    t = torch.from_numpy(np.ascontiguousarray(a)).to(DEV)
    return t if dtype is None else t.to(dtype)


def strided(t, pad):
    """The same matrix with rows `pad` elements apart."""
    if not pad:
        return t
    full = torch.full((t.shape[0], t.shape[1] + pad), 7, dtype=t.dtype, device=t.device)
    full[:, :t.shape[1]] = t
    return full[:, :t.shape[1]]


# ------------------------------------------------------------------------------------------------ quantization
def quantized(ctx, x, mdiag=None, values=None, count=None):
    out = aser.Mx4.empty(x.shape[-2], x.shape[-1], count)
    out.codes.fill_(0xA5)
    out.scales.fill_(0xA5)
    ctx.check(aser.aser_mx4_quantize(ctx, x, out, mdiag=mdiag, values=values))
    return out


def rows_of(t, rows):
    """Panels of scales (panels x words x 16 x 4) or of codes (panels x words x 4 x 16 x 16) as rows x words x bytes."""
    t = t.cpu().numpy()
    t = t.transpose(0, 3, 1, 2, 4) if t.ndim == 5 else t.transpose(0, 2, 1, 3)
    return t.reshape(t.shape[0] * 16, t.shape[2], -1)[:rows]


def check_quantized(x, out, values, mdiag=None):
    codes, scales = orc.quantize(x.float().cpu().numpy(), None if mdiag is None else mdiag.cpu().numpy())
    want_c, want_s = orc.pack(codes, scales)
    rows = x.shape[0]
    assert np.array_equal(rows_of(out.scales, rows), want_s.transpose(1, 0, 2))
    got = rows_of(out.codes, rows).reshape(rows, -1)
    assert np.array_equal(got, want_c), np.argwhere(got != want_c)[:5]
    assert (rows_of(out.codes, None)[rows:] == 0xA5).all() and (rows_of(out.scales, None)[rows:] == 0xA5).all()
    if values is not None:
        v = orc.values(codes, scales)[:, :x.shape[1]]
        assert np.array_equal(values.double().cpu().numpy(), v, equal_nan=True)


@pytest.mark.parametrize("rows,n,dtype,m,pad", [
    (1, 1, torch.float32, False, 0), (1, 4096, torch.bfloat16, True, 0), (3, 31, torch.bfloat16, False, 1), (5, 33, torch.float32, True, 0),
    (17, 128, torch.bfloat16, False, 0), (2, 129, torch.float32, False, 3), (33, 500, torch.bfloat16, True, 4), (40, 1408, torch.float32, True, 8),
    (257, 96, torch.bfloat16, True, 0), (130, 2056, torch.float32, False, 0)])
def test_quantize(ctx, rows, n, dtype, m, pad):
    rng = np.random.default_rng(rows * 1000 + n)
    x = rng.standard_normal((rows, n)) * np.exp2(rng.integers(-12, 12, (rows, (n + 31) // 32)))[:, np.arange(n) // 32]
    x[rng.random((rows, n)) < 0.05] = 0.0
    x = strided(dev(x, dtype), pad)
    mdiag = dev(rng.random(n) * 9 + 0.3, torch.float32) if m else None
    values = strided(torch.zeros(rows, n, dtype=dtype, device=DEV), 2 * pad)
    out = quantized(ctx, x, mdiag, values)
    check_quantized(x, out, values, mdiag)
    again = quantized(ctx, x, mdiag)
    assert torch.equal(again.codes, out.codes) and torch.equal(again.scales, out.scales)
    want = values.clone()
    quantized(ctx, x, mdiag, x)                                    # in place
    assert torch.equal(x, want)


def test_quantize_every_bf16_number(ctx):
    """All 65536 bit patterns, each in blocks whose largest is itself, and in blocks with a larger one of its binade's neighbours."""
    bits = np.arange(65536, dtype=np.uint32)
    x = torch.from_numpy((bits << 16).view(np.float32)).reshape(-1, 1).repeat(1, 64)
    x[:, 1:32] = 0
    for j in range(31):                                            # the block's largest is j eighths of a binade above the number
        x[:, 33 + j] = 0
    x[:, 63] = x[:, 32] * (1.0 + 0.25 * torch.from_numpy((bits % 29).astype(np.float32)))
    x = x.to(torch.bfloat16).to(DEV)
    values = torch.empty_like(x)
    check_quantized(x, quantized(ctx, x, values=values), values)


def test_quantize_ties_borders_and_extremes(ctx):
    ties = np.array([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 7.0, 6.0, 7.999])
    near = np.concatenate([ties, np.nextafter(ties.astype(np.float32), np.float32(0)), np.nextafter(ties.astype(np.float32), np.float32(9))])
    rows = []
    for e in (-149, -140, -130, -127, -126, -125, -124, -60, 0, 60, 120, 125):
        for sign in (1, -1):
            with np.errstate(all="ignore"):
                block = np.float32(sign) * np.ldexp(near.astype(np.float32), e)
            row = np.zeros(32, np.float32)
            row[:30] = np.where(np.isfinite(block), block, 0)
            with np.errstate(all="ignore"):
                row[30] = np.float32(np.ldexp(4.0, e)) if e < 125 else np.float32(3e38)
            rows.append(row)
    zero, neg = np.zeros(32, np.float32), -np.zeros(32, np.float32)
    x = np.concatenate([np.stack(rows + [zero, neg]), np.full((1, 32), 3.4028235e38, np.float32), np.full((1, 32), 1.4e-45, np.float32)])
    for value in (np.inf, -np.inf, np.nan):
        row = np.ones(32, np.float32)
        row[5] = value
        x = np.concatenate([x, row[None]])
    x = np.concatenate([x, x[::-1]], 1)                            # a block beside a NaN block keeps its numbers
    x = dev(x)
    values = torch.empty_like(x)
    check_quantized(x, quantized(ctx, x, values=values), values)


def test_quantize_several_matrices_and_none(ctx):
    x = torch.randn(3, 5, 200, device=DEV)
    values = torch.empty_like(x)
    out = quantized(ctx, x, values=values, count=3)
    for e in range(3):
        one = aser.Mx4(out.codes[e], out.scales[e], 200, 5)
        check_quantized(x[e], one, values[e])
    none = aser.Mx4.empty(0, 64)
    ctx.check(aser.aser_mx4_quantize(ctx, torch.empty(0, 64, device=DEV), none))


# ------------------------------------------------------------------------------------------------ products
def matrix(rng, rows, n, top=2, count=None):
    """A random matrix in 4 bits: (Mx4, its values rows x n in float64)."""
    total = rows * (count or 1)
    x = rng.standard_normal((total, n)) * np.exp2(rng.integers(-top, top + 1, (total, (n + 31) // 32)))[:, np.arange(n) // 32]
    codes, scales = orc.quantize(x)
    v = orc.values(codes, scales)[:, :n]
    if count is None:
        return aser.Mx4(*(dev(a) for a in orc.pack(codes, scales)), n), v
    parts = [orc.pack(codes[i * rows:(i + 1) * rows], scales[i * rows:(i + 1) * rows]) for i in range(count)]
    return aser.Mx4(dev(np.stack([p[0] for p in parts])), dev(np.stack([p[1] for p in parts])), n), v.reshape(count, rows, n)


def factors(rng, m, n, r, count=None):
    front = () if count is None else (count,)
    a, b = (dev(rng.standard_normal(front + s) * q, torch.bfloat16) for s, q in (((m, r), 0.3), ((r, n), n ** -0.5)))
    return a, b, a.double().cpu().numpy(), b.double().cpu().numpy()


def expected(x, w, a, b, swiglu, dtype, r):
    z, size = orc.product(x, w, a, b)
    off = sums_off(x.shape[1], r) * size
    if swiglu:                                                     # silu's slope is below 1.1; its own rounding is a few units of fp32
        m = z.shape[1] // 2
        y = orc.gated(z)
        with np.errstate(over="ignore"):
            silu = np.abs(z[:, :m] / (1 + np.exp(-z[:, :m])))
        off = 1.1 * off[:, :m] * (np.abs(z[:, m:]) + off[:, m:]) + silu * off[:, m:] + np.abs(y) * 16 * 2.0 ** -24
        z = y
    return z, off + rounding(np.abs(z) + off, dtype)


SHAPES = [(1, 1, 1, 0), (1, 31, 3, 1), (1, 4096, 48, 64), (2, 33, 16, 8), (5, 128, 17, 0), (16, 160, 33, 13), (17, 512, 100, 0), (31, 640, 64, 16), (33, 1408, 130, 32),
          (64, 500, 257, 0), (65, 2056, 40, 128), (130, 256, 300, 0), (257, 384, 512, 64), (300, 4128, 258, 24), (515, 130, 770, 100), (700, 1000, 1030, 0),
          # by the numbers of workgroups: other fragments for few rows, both kinds of tiles
          (2, 160, 16390, 20), (61, 130, 12850, 8), (700, 260, 4200, 33), (1000, 130, 16500, 64)]


@pytest.mark.parametrize("swiglu", [False, True], ids=["plain", "gated"])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
@pytest.mark.parametrize("rows,n,m,r", SHAPES)
def test_forward(ctx, rows, n, m, r, dtype, swiglu):
    rng = np.random.default_rng(rows + n + m + r)
    outs, m = m, 2 * m if swiglu else m
    (x, xv), (w, wv) = matrix(rng, rows, n), matrix(rng, m, n)
    a, b, av, bv = factors(rng, m, n, r) if r else (None,) * 4
    ctx.ensure_workspace(aser.aser_mx4_forward_workspace_bytes(rows, n, m, r))
    for pad in (0, 5):
        full = torch.full((rows + 2, outs + pad), 7.0, dtype=dtype, device=DEV)
        y = full[:rows, :outs]
        ctx.check(aser.aser_mx4_forward(ctx, x, w, y, L_A=a, L_B=b, swiglu=swiglu))
        close(y, *expected(xv, wv, av, bv, swiglu, dtype, r))
        assert (full[rows:] == 7).all() and (full[:, outs:] == 7).all()


@pytest.mark.parametrize("swiglu", [False, True], ids=["plain", "gated"])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
@pytest.mark.parametrize("rows,n,m,r", [(2050, 2100, 6210, 0), (1930, 2176, 6660, 40)])
def test_forward_largest_tiles(ctx, rows, n, m, r, dtype, swiglu):
    """Sizes that take tiles of 256 x 256; random codes, the products of the reference on the device, in 64 bits."""
    rng = np.random.default_rng(rows)
    outs, m = m, 2 * m if swiglu else m
    made = []
    for count in (rows, m):
        codes, scales = rng.integers(0, 16, (count, orc.width(n))).astype(np.uint8), rng.integers(124, 128, (count, orc.width(n) // 32)).astype(np.uint8)
        codes[:, n:] = 0
        made.append((aser.Mx4(*(dev(a) for a in orc.pack(codes, scales)), n), dev(orc.values(codes, scales)[:, :n])))
    (x, xv), (w, wv) = made
    a, b, *_ = factors(rng, m, n, r) if r else (None, None)
    z, size = xv @ wv.t(), xv.abs() @ wv.abs().t()
    if r:
        z += (xv @ b.double().t()) @ a.double().t()
        size += (xv.abs() @ b.double().abs().t()) @ a.double().abs().t()
    off = sums_off(n, r) * size
    if swiglu:
        g, u = z[:, :outs], z[:, outs:]
        silu = g * torch.sigmoid(g)
        off = 1.1 * off[:, :outs] * (u.abs() + off[:, outs:]) + silu.abs() * off[:, outs:] + (silu * u).abs() * 16 * 2.0 ** -24
        z = silu * u
    off += (z.abs() + off) * (2.0 ** -8 if dtype == torch.bfloat16 else 2.0 ** -24)
    ctx.ensure_workspace(aser.aser_mx4_forward_workspace_bytes(rows, n, m, r))
    y = torch.full((rows, outs), 7.0, dtype=dtype, device=DEV)
    ctx.check(aser.aser_mx4_forward(ctx, x, w, y, L_A=a, L_B=b, swiglu=swiglu))
    assert ((y.double() - z).abs() <= off).all()


@pytest.mark.parametrize("rows,m", [(1, 300), (20, 300), (40, 300), (300, 300), (700, 4200)])
def test_forward_extreme_scales_and_nan(ctx, rows, m):
    """Blocks of the smallest and largest scales; NaN blocks stay in their rows and outputs."""
    rng = np.random.default_rng(rows)
    n = 256
    xc, wc = rng.integers(0, 16, (rows, n)).astype(np.uint8), rng.integers(0, 16, (m, n)).astype(np.uint8)
    xs, ws = rng.integers(125, 130, (rows, n // 32)).astype(np.uint8), rng.integers(125, 130, (m, n // 32)).astype(np.uint8)
    xs[0, :4], xs[0, 4:] = 0, 1                                    # tokens of 2^-127, weights of 2^100 to 2^125
    ws[0], ws[1], ws[2] = 252, 230, 0
    if rows > 1:
        xs[rows - 1, 3] = 255
        xs[1] = 250
        ws[:, 5] = np.minimum(ws[:, 5], 127)
    ws[7, 2] = 255
    xv, wv = orc.values(xc, xs), orc.values(wc, ws)
    x, w = (aser.Mx4(*(dev(p) for p in orc.pack(c, s)), n) for c, s in ((xc, xs), (wc, ws)))
    r = 16
    a, b, av, bv = factors(rng, m, n, r)
    ctx.ensure_workspace(aser.aser_mx4_forward_workspace_bytes(rows, n, m, r))
    for fa in (None, a):
        y = torch.zeros(rows, m, device=DEV)
        ctx.check(aser.aser_mx4_forward(ctx, x, w, y, L_A=fa, L_B=None if fa is None else b))
        with np.errstate(all="ignore"):
            z, size = orc.product(xv, wv, *((av, bv) if fa is not None else ()))
        top = np.nan_to_num(size, nan=0.0) < 3e38                  # beyond fp32 there is nothing to compare
        got = y.double().cpu().numpy()
        assert (np.isnan(got) == np.isnan(z))[top | np.isnan(z)].all()
        tiny = 2.0 ** -126                                         # sums below the normal numbers may be flushed
        for pad in (0, 3):                                         # the same places are NaN in 16 bits, whatever the rows' alignment
            half = strided(torch.zeros(rows, m, dtype=torch.bfloat16, device=DEV), pad)
            ctx.check(aser.aser_mx4_forward(ctx, x, w, half, L_A=fa, L_B=None if fa is None else b))
            assert torch.equal(half.isnan(), y.isnan())
        ok = np.abs(got - z) <= (sums_off(n, r) + 2.0 ** -24) * size + tiny * (1 + (np.abs(av).sum(1) if fa is not None else 0))
        assert (ok | np.isnan(z) | ~top).all(), np.argwhere(~(ok | np.isnan(z) | ~top))[:5]


# ------------------------------------------------------------------------------------------------ routing
def routed(ctx, logits, k, **opts):
    rows, experts = logits.shape
    plan = aser.ExpertPlan.empty(rows, k, experts)
    for t in (plan.ids, plan.offsets, plan.order, plan.place):
        t.fill_(12345)
    plan.weights.fill_(float("nan"))
    ctx.ensure_workspace(aser.aser_route_workspace_bytes(rows, experts, k))
    ctx.check(aser.aser_route_experts(ctx, logits, plan, **opts))
    return plan


def check_routed(logits, plan, k, **opts):
    opts["bias"] = None if opts.get("bias") is None else opts["bias"].double().cpu().numpy()
    ids, weights = orc.route(logits.double().cpu().numpy(), k, **opts)
    offsets, order, place = orc.plan(ids, logits.shape[1])
    assert np.array_equal(plan.ids.cpu().numpy(), ids)
    got = plan.weights.double().cpu().numpy()
    assert (np.abs(got - weights) <= np.abs(weights) * (2.0 ** -24 + 1e-12) + 2.0 ** -149).all()
    assert np.array_equal(plan.offsets.cpu().numpy(), offsets)
    assert np.array_equal(plan.order.cpu().numpy(), order)
    assert np.array_equal(plan.place.cpu().numpy(), place)


ROUTES = [
    (1, 1, 1, {}), (1, 64, 6, {}), (3, 8, 8, dict(sigmoid=True)), (31, 60, 4, dict(renormalize=False)), (32, 64, 6, dict(sigmoid=True, bias=True, scale=2.5)),
    (33, 65, 5, dict(bias=True)), (64, 128, 32, dict(sigmoid=True, renormalize=False)), (100, 256, 8, dict(sigmoid=True, bias=True, groups=8, top_groups=4, group_top=2)),
    (65, 160, 6, dict(groups=8, top_groups=3)), (40, 16, 8, dict(groups=4, top_groups=1, group_top=2)), (129, 512, 9, dict(groups=64, top_groups=5, group_top=2)),
    (70, 1000, 12, dict(bias=True)), (35, 1024, 7, dict(sigmoid=True, groups=2, top_groups=1, group_top=2)), (2100, 8, 2, {}), (500, 384, 8, dict(sigmoid=True, bias=True)),
    (64, 48, 3, dict(groups=48, top_groups=7, group_top=2, bias=True))]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
@pytest.mark.parametrize("rows,experts,k,opts", ROUTES)
def test_route(ctx, rows, experts, k, opts, dtype):
    g = torch.Generator().manual_seed(rows + experts)
    logits = (torch.randn(rows, experts, generator=g) * 2).to(DEV, dtype)
    opts = dict(opts)
    if opts.get("bias"):
        opts["bias"] = (torch.randn(experts, generator=g) * 0.1).to(DEV)
    logits = strided(logits, 3)
    check_routed(logits, routed(ctx, logits, k, **opts), k, **opts)


@pytest.mark.parametrize("sigmoid", [False, True])
@pytest.mark.parametrize("bias", [False, True])
@pytest.mark.parametrize("rows", [7, 80])
def test_route_ties_masks_and_values_that_are_none(ctx, rows, bias, sigmoid):
    inf = float("inf")
    g = torch.Generator().manual_seed(3)
    logits = torch.randint(-2, 3, (rows, 24), generator=g).float()               # many ties
    logits[0] = -inf                                                             # nothing to choose
    logits[1, 1:] = -inf                                                         # one expert
    logits[2, 5:] = float("nan")
    logits[3, 4], logits[3, 9] = inf, inf
    logits[4] = 200.0                                                            # all alike, saturated
    logits[5] = -200.0
    logits[6] = torch.arange(24).float() * 40 - 480                              # from e^-480 to e^480
    logits = logits.to(DEV)
    b = (torch.randint(-1, 2, (24,), generator=g).float() * 0.25).to(DEV) if bias else None
    for opts in (dict(), dict(groups=4, top_groups=2, group_top=2), dict(groups=6, top_groups=5), dict(renormalize=False)):
        opts = dict(opts, bias=b, sigmoid=sigmoid)
        check_routed(logits, routed(ctx, logits, 6, **opts), 6, **opts)
    if bias:
        b[3], b[4], b[5] = float("nan"), -inf, inf
        opts = dict(bias=b, sigmoid=sigmoid)
        check_routed(logits, routed(ctx, logits, 6, **opts), 6, **opts)


# 33 rows and more, around the widths, choices and groups up to which 16 lanes have a row; few different logits, so that experts tie within and across lanes
@pytest.mark.parametrize("rows", [33, 97])
@pytest.mark.parametrize("sigmoid", [False, True])
@pytest.mark.parametrize("experts,k,opts", [
    (16, 16, dict()), (17, 3, dict(renormalize=False)), (64, 16, dict(groups=16, top_groups=7, group_top=2)), (65, 17, dict()), (66, 4, dict(groups=33, top_groups=8)),
    (128, 8, dict(groups=4, top_groups=2, group_top=2)), (129, 5, dict(groups=3, top_groups=2)), (255, 15, dict(groups=15, top_groups=4, group_top=2, bias=True)),
    (256, 16, dict(bias=True)), (256, 32, dict()), (256, 8, dict(groups=2, top_groups=1)), (257, 6, dict(bias=True)),
    (384, 8, dict(groups=8, top_groups=4, group_top=2, bias=True)), (385, 4, dict())])
def test_route_many_rows_with_ties(ctx, rows, sigmoid, experts, k, opts):
    g = torch.Generator().manual_seed(rows + experts + k)
    logits = torch.randint(-3, 4, (rows, experts), generator=g).float()
    logits[rows // 2] = -float("inf")
    logits[rows - 1, k // 2:] = -float("inf")
    logits[:, experts - 1] = float("nan")
    opts = dict(opts, sigmoid=sigmoid)
    if opts.get("bias"):
        opts["bias"] = (torch.randint(-1, 2, (experts,), generator=g).float() * 0.25).to(DEV)
    logits = logits.to(DEV)
    check_routed(logits, routed(ctx, logits, k, **opts), k, **opts)


# rows whose logits all lie where 64 bits end: exp(-l) is finite down to -709.78265380859375 in 32 bits, infinite from the next number on
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
@pytest.mark.parametrize("sigmoid", [False, True])
@pytest.mark.parametrize("rows", [19, 80])
def test_route_far_below_zero(ctx, rows, sigmoid, dtype):
    lowest = float(torch.finfo(dtype).min)
    far = [-700.0, -705.0, -708.0, -709.5, -709.78265380859375, -709.78271484375, -710.0, -712.0, -715.0, -720.0, -725.0, -730.0, -736.0, -740.0, -744.0, -745.0, -746.0, -750.0,
           -760.0, -1e3, -1e4, -1e9, -3e38, lowest]
    experts = len(far)
    logits = torch.full((rows, experts), lowest)
    g = torch.Generator().manual_seed(rows)
    logits[0] = torch.tensor(far)
    logits[1] = torch.tensor(far)[torch.randperm(experts, generator=g)]
    logits[2, 4:12] = torch.tensor([-720.0, -730.0, -740.0, -715.0, -716.0, -717.0, -718.0, -719.0])
    logits[3] = torch.arange(experts) * -2.0 - 690.0
    logits[4] = -1e9
    logits[5] = torch.arange(experts) * -1e4 - 1e4
    logits[6] = torch.tensor(far)
    logits[6, 3::5] = torch.arange(5) * 1.5 - 2.0                                # ordinary ones among them
    logits[7] = -709.0
    logits[8] = -float("inf")
    logits[8, :4] = torch.tensor([-705.0, -715.0, -1000.0, lowest])
    logits[9, :2] = 3.0                                                          # the rest is masked with the lowest number, and some of it has to be chosen
    for t in range(11, rows):
        logits[t] = torch.tensor(far)[torch.randint(0, experts, (experts,), generator=g)]        # row 10 is masked altogether
    logits = logits.to(dtype).to(DEV)
    b = (torch.randint(-1, 2, (experts,), generator=g).float() * 0.25).to(DEV)
    for bias in (None, b):
        for opts in (dict(), dict(renormalize=False), dict(groups=4, top_groups=2, group_top=2), dict(groups=6, top_groups=3)):
            opts = dict(opts, bias=bias, sigmoid=sigmoid, scale=2.5)
            check_routed(logits, routed(ctx, logits, 6, **opts), 6, **opts)


def test_route_scale_that_is_changed_in_place(ctx):
    logits, scale = torch.randn(5, 8, generator=torch.Generator().manual_seed(2)).to(DEV), torch.tensor(2.0)
    for value in (2.0, 3.0):
        scale.fill_(value)
        plan = routed(ctx, logits, 2, scale=scale)
        check_routed(logits, plan, 2, scale=value)


def test_route_no_rows(ctx):
    plan = aser.ExpertPlan.empty(0, 2, 300)
    plan.offsets.fill_(9)
    ctx.check(aser.aser_route_experts(ctx, torch.empty(0, 300, device=DEV), plan))
    assert (plan.offsets == 0).all()


# ------------------------------------------------------------------------------------------------ the experts' products
def given_plan(rng, rows, k, experts, drop=0.0, skew=0.0):
    """A plan of random choices; some pairs have no expert, and with skew some experts get most rows."""
    ids = np.stack([rng.choice(experts, k, replace=False, p=None if not skew else (lambda p: p / p.sum())(np.exp(-skew * np.arange(experts)))) for _ in range(rows)])
    ids[rng.random(ids.shape) < drop] = -1
    offsets, order, place = orc.plan(ids, experts)
    i32 = lambda a: dev(a.astype(np.int32))                        # noqa: E731
    weights = rng.random((rows, k)).astype(np.float32)
    return aser.ExpertPlan(i32(ids), dev(weights), i32(offsets), i32(order), i32(place)), ids, weights, offsets, order, place


EXPERTS = [(1, 8, 2, 256, 48, 0, 0, 0), (1, 4, 4, 40, 17, 5, 0, 0), (3, 100, 6, 128, 16, 0, 0, 0), (16, 64, 6, 256, 40, 16, 0.1, 0), (40, 5, 3, 1408, 36, 0, 0, 1.0),
           (100, 8, 2, 384, 130, 32, 0.3, 0), (300, 3, 1, 200, 260, 0, 0, 2.0), (260, 4, 2, 512, 258, 64, 0, 0), (1000, 16, 4, 128, 64, 8, 0.5, 0.3), (200, 130, 2, 160, 33, 0, 0, 0),
           # by the numbers of workgroups: other fragments for few rows, both kinds of tiles
           (640, 256, 8, 128, 264, 8, 0, 0), (1280, 256, 8, 100, 264, 0, 0, 0), (1700, 256, 8, 96, 40, 16, 0, 0), (1500, 4, 2, 256, 1100, 64, 0.1, 0.5),
           (1200, 5, 2, 130, 6200, 5, 0, 0.3), (700, 1, 1, 256, 4200, 32, 0.2, 0), (30, 1, 1, 130, 50, 0, 0, 0)]


@pytest.mark.parametrize("gather,swiglu", [(True, True), (False, False), (True, False)], ids=["up", "down", "gather"])
@pytest.mark.parametrize("rows,experts,k,n,m,r,drop,skew", EXPERTS)
def test_expert_forward(ctx, rows, experts, k, n, m, r, drop, skew, gather, swiglu):
    rng = np.random.default_rng(rows + experts + n)
    dtype = torch.float32 if (rows + k) % 2 else torch.bfloat16
    outs, m = m, 2 * m if swiglu else m
    plan, ids, _, offsets, order, _ = given_plan(rng, rows, k, experts, drop, skew)
    (x, xv), (w, wv) = matrix(rng, rows if gather else rows * k, n), matrix(rng, m, n, count=experts)
    a, b, av, bv = factors(rng, m, n, r, experts) if r else (None,) * 4
    ctx.ensure_workspace(aser.aser_expert_forward_workspace_bytes(rows * k, n, m, experts, r))
    y = torch.full((rows * k, outs), 7.0, dtype=dtype, device=DEV)
    ctx.check(aser.aser_expert_forward(ctx, x, w, plan, y, gather=gather, L_A=a, L_B=b, swiglu=swiglu))
    for e in range(experts):
        here = slice(offsets[e], offsets[e + 1])
        if offsets[e] == offsets[e + 1]:
            continue
        mine = xv[order[here] // k] if gather else xv[here]
        close(y[here], *expected(mine, wv[e], None if av is None else av[e], None if bv is None else bv[e], swiglu, dtype, r))
    assert (y[offsets[-1]:] == 7).all()


def test_experts_plan_is_not_trusted(ctx):
    """Offsets and orders that make no sense are clamped: the call ends and writes inside Y alone."""
    rng = np.random.default_rng(5)
    plan, *_ = given_plan(rng, 20, 2, 4)
    (x, _), (w, _) = matrix(rng, 20, 128), matrix(rng, 32, 128, count=4)
    full = torch.full((60, 32), 7.0, device=DEV)
    for offsets in ([0, 1000, -5, 2 ** 31 - 1, 40], [40, 30, 20, 10, 0], [-2 ** 31, 2 ** 31 - 1, 0, 7, 2 ** 31 - 1]):
        plan.offsets.copy_(torch.tensor(offsets, dtype=torch.int64).to(torch.int32))
        plan.order.copy_(torch.randint(-2 ** 31, 2 ** 31 - 1, (40,)).to(torch.int32))
        plan.place.copy_(torch.randint(-2 ** 31, 2 ** 31 - 1, (40,)).to(torch.int32))
        ctx.check(aser.aser_expert_forward(ctx, x, w, plan, full[10:50], gather=True))
        out = torch.zeros(20, 32, device=DEV)
        ctx.check(aser.aser_expert_combine(ctx, full[10:50], plan, out))
        assert (full[:10] == 7).all() and (full[50:] == 7).all()


@pytest.mark.parametrize("gather", [True, False])
@pytest.mark.parametrize("rows,experts,m,r", [(900, 3, 2400, 0), (900, 3, 2400, 40), (1500, 20, 4200, 0), (1500, 20, 4200, 24)])
def test_experts_plan_is_not_trusted_with_many_rows(ctx, rows, experts, m, r, gather):
    """The same for tiles: their numbering, the rows put in order, P and its terms."""
    rng = np.random.default_rng(rows + r)
    k, n = 2, 256
    pairs = rows * k
    plan, *_ = given_plan(rng, rows, k, experts)
    x, w = aser.Mx4.empty(rows if gather else pairs, n), aser.Mx4.empty(m, n, experts)
    for t in (x, w):
        t.codes.random_(0, 256)
        t.scales.random_(120, 130)
    a, b, *_ = factors(rng, m, n, r, experts) if r else (None,) * 4
    ctx.ensure_workspace(aser.aser_expert_forward_workspace_bytes(pairs, n, m, experts, r))
    full = torch.full((pairs + 600, m), 7.0, device=DEV, dtype=torch.bfloat16)
    ends = [2 ** 31 - 1, -2 ** 31, 0, pairs, pairs - 1, 7, -1, pairs + 1, pairs // 2]
    for offsets in (rng.integers(-2 ** 31, 2 ** 31, experts + 1), rng.choice(ends, experts + 1), np.sort(rng.integers(0, pairs + 1, experts + 1))[::-1], np.resize([0, 2 ** 31 - 1], experts + 1)):
        plan.offsets.copy_(dev(offsets.astype(np.int32)))
        plan.order.copy_(dev(rng.integers(-2 ** 31, 2 ** 31, pairs).astype(np.int32)))
        ctx.check(aser.aser_expert_forward(ctx, x, w, plan, full[300:300 + pairs], gather=gather, L_A=a, L_B=b))
        assert (full[:300] == 7).all() and (full[300 + pairs:] == 7).all()


# ------------------------------------------------------------------------------------------------ the weighted sum
@pytest.mark.parametrize("rows,k,m,y_type,out_type,pad,base", [
    (1, 1, 1, torch.float32, torch.float32, 0, "none"), (1, 6, 2048, torch.bfloat16, torch.bfloat16, 0, "none"), (7, 2, 100, torch.bfloat16, torch.float32, 3, "other"),
    (33, 8, 4104, torch.float32, torch.bfloat16, 0, "same"), (50, 3, 2049, torch.bfloat16, torch.bfloat16, 8, "other"), (9, 32, 72, torch.float32, torch.float32, 0, "same")])
def test_combine(ctx, rows, k, m, y_type, out_type, pad, base):
    rng = np.random.default_rng(rows + m)
    plan, ids, weights, _, _, place = given_plan(rng, rows, k, 32, drop=0.2)
    y = strided(dev(rng.standard_normal((rows * k, m)), y_type), pad)
    y[plan.offsets[-1].item():] = float("nan")                     # nobody looks there
    out = strided(dev(rng.standard_normal((rows, m)), out_type), pad)
    y0 = None if base == "none" else out if base == "same" else strided(dev(rng.standard_normal((rows, m)), out_type), pad)
    want = np.zeros((rows, m)) if y0 is None else y0.double().cpu().numpy()
    size = np.abs(want)
    yv = y.double().cpu().numpy()
    for t in range(rows):
        for j in range(k):
            if ids[t, j] >= 0:
                term = float(weights[t, j]) * yv[place[t * k + j]]
                want[t] += term
                size[t] += np.abs(term)
    ctx.check(aser.aser_expert_combine(ctx, y, plan, out, Y0=y0))
    off = (k + 1) * 2.0 ** -24 * size
    close(out, want, off + rounding(np.abs(want) + off, out_type))


# ------------------------------------------------------------------------------------------------ together
class Layer:
    """A layer of experts on fixed buffers: what a decoding server replays."""

    def __init__(self, ctx, rng, rows, experts, k, n, m, r):
        self.ctx, self.rows, self.n = ctx, rows, n
        self.up, self.up_v = matrix(rng, 2 * m, n, count=experts)
        self.down, self.down_v = matrix(rng, n, m, count=experts)
        self.a, self.b, self.av, self.bv = factors(rng, 2 * m, n, r, experts)
        self.router = dev(rng.standard_normal((n, experts)) * 0.05, torch.float32)
        self.x = torch.zeros(rows, n, dtype=torch.bfloat16, device=DEV)
        self.logits = torch.zeros(rows, experts, device=DEV)
        self.plan = aser.ExpertPlan.empty(rows, k, experts)
        self.xq, self.hq = aser.Mx4.empty(rows, n), aser.Mx4.empty(rows * k, m)
        self.h = torch.zeros(rows * k, m, dtype=torch.bfloat16, device=DEV)
        self.y = torch.zeros(rows * k, n, dtype=torch.bfloat16, device=DEV)
        self.out = torch.zeros(rows, n, dtype=torch.bfloat16, device=DEV)
        for need in (aser.aser_route_workspace_bytes(rows, experts, k), aser.aser_expert_forward_workspace_bytes(rows * k, n, 2 * m, experts, r),
                     aser.aser_expert_forward_workspace_bytes(rows * k, m, n, experts, 0)):
            ctx.ensure_workspace(need)

    def step(self):
        c = self.ctx
        c.check(aser.aser_route_experts(c, self.logits, self.plan, sigmoid=True))
        c.check(aser.aser_mx4_quantize(c, self.x, self.xq))
        c.check(aser.aser_expert_forward(c, self.xq, self.up, self.plan, self.h, gather=True, swiglu=True, L_A=self.a, L_B=self.b))
        c.check(aser.aser_mx4_quantize(c, self.h, self.hq))
        c.check(aser.aser_expert_forward(c, self.hq, self.down, self.plan, self.y, gather=False))
        c.check(aser.aser_expert_combine(c, self.y, self.plan, self.out))

    def give(self, rng):
        x = dev(rng.standard_normal((self.rows, self.n)), torch.bfloat16)
        self.x.copy_(x)
        self.logits.copy_(x.float() @ self.router)
        self.logits[self.rows // 2, 1:] = float("-inf")                          # one row has one expert only
        return x


@pytest.mark.parametrize("rows,experts,k,n,m,r", [(3, 8, 2, 256, 96, 16), (40, 6, 3, 384, 200, 32), (900, 4, 2, 256, 2100, 32)])
def test_layer_replayed_on_another_stream(rows, experts, k, n, m, r):
    """A captured layer gives the eager results' bits on every replay, with other inputs, eager work and other streams' work between them."""
    rng = np.random.default_rng(rows)
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        layer = Layer(aser.Context(0, side.cuda_stream), rng, rows, experts, k, n, m, r)
        eager = Layer(aser.Context(0, side.cuda_stream), np.random.default_rng(rows), rows, experts, k, n, m, r)
        layer.give(rng)
        layer.step()
        side.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            layer.step()
        other = aser.Context(0, torch.cuda.current_stream().cuda_stream)
        for rep in range(4):
            seed = 100 * rows + rep
            layer.give(np.random.default_rng(seed))
            eager.give(np.random.default_rng(seed))
            graph.replay()
            eager.step()
            side.synchronize()
            assert torch.equal(layer.out, eager.out) and torch.equal(layer.plan.order, eager.plan.order)
            used = int(layer.plan.offsets[-1])
            assert torch.equal(layer.h[:used], eager.h[:used]) and used == rows * k - (k - 1)
            quantized(other, layer.x)
    assert layer.out.isfinite().all() and layer.out.abs().max() > 0


@pytest.mark.parametrize("rows,experts,k,n,m,r", [(40, 6, 3, 384, 200, 32), (900, 4, 2, 256, 2100, 32)])
def test_layer_replayed_beside_another_streams_work(rows, experts, k, n, m, r):
    """Replays while another stream runs an eager layer of its own, with no wait between the two: both have the bits of quiet runs."""
    side, other = torch.cuda.Stream(), torch.cuda.Stream()
    layers = []
    for stream, seed in ((side, rows), (other, rows + 1)):
        with torch.cuda.stream(stream):
            layers.append(Layer(aser.Context(0, stream.cuda_stream), np.random.default_rng(seed), rows, experts, k, n, m, r))
            layers[-1].give(np.random.default_rng(seed + 50))
            layers[-1].step()
    torch.cuda.synchronize()
    want = [layer.out.clone() for layer in layers]
    captured, eager = layers
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        captured.step()
    for rep in range(6):
        torch.cuda.synchronize()
        for layer in layers:
            layer.out.zero_()
        torch.cuda.synchronize()
        for _ in range(3):
            with torch.cuda.stream(side):
                graph.replay()
            with torch.cuda.stream(other):
                eager.step()
        torch.cuda.synchronize()
        for layer, out in zip(layers, want):
            assert torch.equal(layer.out, out), rep


def test_two_contexts_at_once():
    """Two layers on streams of their own, enqueued without a wait between them, have the results that each has alone."""
    sizes = [(33, 8, 2, 256, 128, 16), (700, 4, 2, 128, 1500, 8)]
    streams = [torch.cuda.Stream() for _ in sizes]
    layers = []
    for i, (s, size) in enumerate(zip(streams, sizes)):
        with torch.cuda.stream(s):
            layers.append(Layer(aser.Context(0, s.cuda_stream), np.random.default_rng(i), *size))
            layers[-1].give(np.random.default_rng(i + 10))
    alone = []
    for layer in layers:
        torch.cuda.synchronize()
        layer.step()
        torch.cuda.synchronize()
        alone.append(layer.out.clone())
    for layer in layers:
        layer.out.zero_()
    torch.cuda.synchronize()
    for _ in range(5):
        for layer in layers:
            layer.step()
    torch.cuda.synchronize()
    for layer, want in zip(layers, alone):
        assert torch.equal(layer.out, want)


def test_calibrated_layer_in_four_bits():
    """The quantizer between aser_smoothed_weight and aser_quant_target, then the compensated layer on its codes: with the factors the layer's outputs are nearer to
    the weight's own than without, and as near as the oracle's product of the same codes and factors is."""
    from gpu_util import new_ctx
    ctx, rng = new_ctx(), np.random.default_rng(7)
    m, n, r, f, tokens = 320, 512, 32, 8, 2048
    W = dev(rng.standard_normal((m, n)) * 0.02, torch.float32)
    x = rng.standard_normal((tokens, n))
    x[:, rng.permutation(n)[:8]] *= 30.0
    X = dev(x, torch.bfloat16)
    buf = aser.LayerBuffers(m, n, r, f, 4, False)
    ctx.ensure_workspace(aser.aser_workspace_bytes(m, n, r))
    ctx.check(aser.aser_gram_accumulate(ctx, X, buf.G, buf.abs_sum, buf.count))
    ctx.check(aser.aser_smooth_outliers(ctx, W, buf.abs_sum, buf.count, f, buf.idx, buf.mdiag))
    Wq, w = torch.empty_like(W), aser.Mx4.empty(m, n)
    ctx.check(aser.aser_smoothed_weight(ctx, W, buf.idx, f, Wq))
    ctx.check(aser.aser_mx4_quantize(ctx, Wq, w, values=Wq))
    ctx.check(aser.aser_quant_target(ctx, W, buf.mdiag, Wq, buf.T))
    st, info = aser.aser_whiten(ctx, buf.G, buf.mdiag, 0.0, buf.S)
    ctx.check(st)
    st, err, _ = aser.aser_error_reconstruct(ctx, buf.T, buf.S, r, buf.L_A, buf.L_B, buf.sigma, idx=buf.idx, f=f)
    ctx.check(st)
    assert info == 0
    L_A, L_B = buf.L_A.to(torch.bfloat16), buf.L_B.to(torch.bfloat16)
    ctx.ensure_workspace(aser.aser_mx4_forward_workspace_bytes(200, n, m, r))
    xq, values, y, bare = aser.Mx4.empty(200, n), torch.empty(200, n, dtype=torch.bfloat16, device=DEV), torch.empty(200, m, device=DEV), torch.empty(200, m, device=DEV)
    ctx.check(aser.aser_mx4_quantize(ctx, X[:200], xq, mdiag=buf.mdiag, values=values))
    ctx.check(aser.aser_mx4_forward(ctx, xq, w, y, L_A=L_A, L_B=L_B))
    ctx.check(aser.aser_mx4_forward(ctx, xq, w, bare))
    f64 = lambda t: t.double().cpu().numpy()                                     # noqa: E731
    close(y, *expected(f64(values), f64(Wq), f64(L_A), f64(L_B), False, torch.float32, r))
    # the same tokens through the weight: smoothing moves the outlier channels' share from the codes to the factors
    want = f64(values) * f64(buf.mdiag) @ f64(W).T
    assert np.linalg.norm(f64(y) - want) < 0.5 * np.linalg.norm(f64(bare) - want)


# ------------------------------------------------------------------------------------------------ more workgroups than a dimension of a launch takes threads for
def test_combine_more_than_2_to_the_24_rows(ctx):
    rows, m = 2 ** 24 + 5, 8
    y = torch.randint(-100, 100, (rows, m), device=DEV, dtype=torch.int32).to(torch.bfloat16)
    place = torch.arange(rows - 1, -1, -1, device=DEV, dtype=torch.int32)
    weights = torch.randint(1, 3, (rows, 1), device=DEV, dtype=torch.int32).float()
    plan = aser.ExpertPlan(torch.zeros(rows, 1, device=DEV, dtype=torch.int32), weights, torch.tensor([0, rows], device=DEV, dtype=torch.int32), place, place)
    out = torch.full((rows, m), 7.0, device=DEV)
    ctx.check(aser.aser_expert_combine(ctx, y, plan, out))
    assert torch.equal(out, y.flip(0).float() * weights)


def test_quantize_more_than_2_to_the_24_panels(ctx):
    rows, count = 2 ** 27 - 11, 3
    x = torch.randint(-4, 5, (count, rows, 1), device=DEV, dtype=torch.int8).to(torch.bfloat16)
    out, values = aser.Mx4.empty(rows, 1, count), torch.full((count, rows, 1), 7.0, device=DEV, dtype=torch.bfloat16)
    ctx.check(aser.aser_mx4_quantize(ctx, x, out, values=values))
    assert torch.equal(values, x)                                  # one number alone in its block is kept
    for e in range(count):
        for at, here in ((0, 16), (2 ** 22, 16), (rows // 16, rows % 16)):
            want, _ = orc.quantize(x[e, 16 * at:16 * at + here].float().cpu().numpy())
            assert np.array_equal(out.codes[e, at, 0, 0, :here, 0].cpu().numpy() & 15, want[:, 0])
