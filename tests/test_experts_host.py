"""Host-side checks of the entry points for layers in microscaled 4 bits and layers of experts: what they refuse, before any HIP call is made."""
import ctypes

import pytest

import paper_2411_07762_amd as aser

P = 0x7F0000001000  # a fake, aligned "device address": validation must fail before it is touched
ARG, SHAPE, DTYPE, ROOM = aser.ASER_ERR_INVALID_ARG, aser.ASER_ERR_SHAPE, aser.ASER_ERR_DTYPE, aser.ASER_ERR_WORKSPACE


@pytest.fixture(scope="module")
def ctx():
    lib = aser.load_library()
    h = ctypes.c_void_p()
    assert lib.aser_create(ctypes.byref(h), 0, None) == aser.ASER_OK
    c = aser.Context.__new__(aser.Context)
    c._lib, c.handle, c.device, c._ws, c._ws_bytes = lib, h, 0, None, 0
    yield c
    c.close()


def mx(rows=40, n=256, count=1, codes=P, scales=P):
    return ctypes.byref(aser.aser_mx4(codes, scales, rows, n, count))


def plan(rows=40, top_k=2, n_experts=8, ids=P, weights=P, offsets=P, order=P, place=P):
    return ctypes.byref(aser.aser_expert_plan(ids, weights, offsets, order, place, rows, top_k, n_experts))


BAD_MATRIX = [(dict(codes=None), ARG), (dict(scales=None), ARG), (dict(codes=P + 8), ARG), (dict(scales=P + 4), ARG), (dict(rows=-1), SHAPE), (dict(n=0), SHAPE),
              (dict(n=(1 << 22) + 1), SHAPE), (dict(rows=(1 << 27) + 1), SHAPE), (dict(count=0), SHAPE), (dict(count=65537), SHAPE), (dict(rows=1 << 20, count=2048), SHAPE)]
BAD_PLAN = [(dict(rows=-1), SHAPE), (dict(top_k=0), SHAPE), (dict(top_k=33, n_experts=64), SHAPE), (dict(top_k=9), SHAPE), (dict(n_experts=0), SHAPE),
            (dict(n_experts=1025), SHAPE), (dict(rows=1 << 26), SHAPE), (dict(offsets=P + 2), ARG), (dict(order=P + 1), ARG)]


def quantize(ctx, out, X=P, dt=1, ldx=256, m=None, values=None, ldv=256):
    return ctx._lib.aser_mx4_quantize(ctx.handle, X, dt, ldx, m, out, values, ldv)


def forward(ctx, x=None, w=None, a=None, b=None, r=0, swiglu=0, Y=P, dt=0, ldy=48):
    return ctx._lib.aser_mx4_forward(ctx.handle, x or mx(), w or mx(48), a, b, r, swiglu, Y, dt, ldy)


def expert(ctx, x=None, w=None, p=None, gather=1, a=None, b=None, r=0, swiglu=0, Y=P, dt=0, ldy=48):
    return ctx._lib.aser_expert_forward(ctx.handle, x or mx(), w or mx(48, count=8), p or plan(), gather, a, b, r, swiglu, Y, dt, ldy)


def route(ctx, p=None, logits=P, dt=1, ldl=8, bias=None, opts=(0, 1, 1, 1, 1, 1.0)):
    return ctx._lib.aser_route_experts(ctx.handle, logits, dt, ldl, bias, ctypes.byref(aser.aser_route_opts(*opts)) if opts else None, p or plan())


def combine(ctx, p=None, Y=P, dt=0, ldy=64, m=64, Y0=None, ldy0=64, out=P + 4096, out_dt=0, ldo=64):
    return ctx._lib.aser_expert_combine(ctx.handle, Y, dt, ldy, m, p or plan(), Y0, ldy0, out, out_dt, ldo)


def test_matrices_are_checked(ctx):
    for kw, status in BAD_MATRIX:
        assert quantize(ctx, mx(**kw)) == status, kw
        assert forward(ctx, x=mx(**kw)) == status, kw
        assert forward(ctx, w=mx(**kw)) == status, kw
        assert expert(ctx, x=mx(**kw)) == status, kw
        assert expert(ctx, w=mx(**dict(dict(rows=48, count=8), **kw))) == status, kw
    assert ctx._lib.aser_mx4_forward(ctx.handle, None, mx(48), None, None, 0, 0, P, 0, 48) == ARG
    assert ctx._lib.aser_mx4_quantize(ctx.handle, P, 1, 256, None, None, None, 0) == ARG
    assert ctx._lib.aser_mx4_forward(None, mx(), mx(48), None, None, 0, 0, P, 0, 48) == ARG
    assert "null" in ctx.last_error()


def test_plans_are_checked(ctx):
    for kw, status in BAD_PLAN:
        assert route(ctx, plan(**kw), ldl=2000) == status, kw
        assert combine(ctx, plan(**kw)) == status, kw
        assert expert(ctx, p=plan(**kw)) == status, kw
    assert ctx._lib.aser_expert_forward(ctx.handle, mx(), mx(48, count=8), None, 1, None, None, 0, 0, P, 0, 48) == ARG


@pytest.mark.parametrize("kw,status", [
    (dict(dt=2), DTYPE), (dict(X=None), ARG), (dict(X=P + 2), ARG), (dict(ldx=255), SHAPE), (dict(values=P, ldv=255), SHAPE), (dict(values=P + 1), ARG), (dict(m=P + 2), ARG),
    (dict(values=P, ldx=260, ldv=256), SHAPE)])
def test_quantize_refuses(ctx, kw, status):
    assert quantize(ctx, mx(), **kw) == status


@pytest.mark.parametrize("kw,status", [
    (dict(dt=2), DTYPE), (dict(x=mx(n=128)), SHAPE), (dict(x=mx(count=2)), SHAPE), (dict(w=mx(48, count=2)), SHAPE), (dict(w=mx(0)), SHAPE), (dict(r=-1), SHAPE),
    (dict(r=129, a=P, b=P), SHAPE), (dict(r=8), ARG), (dict(r=8, a=P), ARG), (dict(r=8, a=P + 1, b=P), ARG), (dict(w=mx(49), ldy=49, swiglu=1), SHAPE), (dict(ldy=47), SHAPE),
    (dict(Y=P + 1), ARG), (dict(Y=P + 2, dt=1), ARG), (dict(Y=None), ARG), (dict(r=8, a=P, b=P), ROOM)])
def test_forward_refuses(ctx, kw, status):
    assert forward(ctx, **kw) == status


@pytest.mark.parametrize("kw,status", [
    (dict(w=mx(48, count=7)), SHAPE), (dict(x=mx(41)), SHAPE), (dict(gather=0), SHAPE), (dict(p=plan(offsets=None)), ARG), (dict(p=plan(order=None)), ARG), (dict(dt=3), DTYPE),
    (dict(ldy=40), SHAPE), (dict(Y=None), ARG), (dict(r=4, a=P, b=P), ROOM), (dict(x=mx(4000), p=plan(4000), w=mx(4800, count=8), ldy=4800), ROOM)])
def test_expert_forward_refuses(ctx, kw, status):
    assert expert(ctx, **kw) == status


@pytest.mark.parametrize("kw,status", [
    (dict(opts=None), ARG), (dict(dt=2), DTYPE), (dict(logits=None), ARG), (dict(logits=P + 2), ARG), (dict(bias=P + 2), ARG), (dict(ldl=7), SHAPE),
    (dict(opts=(0, 0, 1, 1, 1, 1.0)), SHAPE), (dict(opts=(0, 3, 1, 1, 1, 1.0)), SHAPE), (dict(opts=(0, 4, 5, 1, 1, 1.0)), SHAPE), (dict(opts=(0, 4, 0, 1, 1, 1.0)), SHAPE),
    (dict(opts=(0, 4, 2, 3, 1, 1.0)), SHAPE), (dict(opts=(0, 1, 1, 1, 1, float("nan"))), ARG), (dict(p=plan(ids=None)), ARG), (dict(p=plan(offsets=None)), ARG),
    (dict(p=plan(place=None)), ARG), (dict(p=plan(n_experts=130), opts=(0, 65, 1, 1, 1, 1.0), ldl=130), SHAPE), (dict(), ROOM)])
def test_route_refuses(ctx, kw, status):
    assert route(ctx, **kw) == status


@pytest.mark.parametrize("kw,status", [
    (dict(dt=2), DTYPE), (dict(out_dt=-1), DTYPE), (dict(Y=None), ARG), (dict(out=None), ARG), (dict(m=0), SHAPE), (dict(ldy=63), SHAPE), (dict(ldo=63), SHAPE),
    (dict(Y0=P, ldy0=63), SHAPE), (dict(Y0=P + 4096, ldy0=65), SHAPE), (dict(Y=P + 1), ARG), (dict(out=P + 2, out_dt=1), ARG), (dict(p=plan(place=None)), ARG),
    (dict(p=plan(weights=None)), ARG)])
def test_combine_refuses(ctx, kw, status):
    assert combine(ctx, **kw) == status


def test_empty_calls_are_no_ops(ctx):
    assert quantize(ctx, mx(0, codes=None, scales=None), X=None) == aser.ASER_OK
    assert forward(ctx, x=mx(0, codes=None, scales=None), Y=None) == aser.ASER_OK
    assert expert(ctx, x=mx(0, codes=None, scales=None), p=plan(0, ids=None, weights=None, offsets=None, order=None, place=None), Y=None) == aser.ASER_OK
    assert combine(ctx, plan(0, ids=None, weights=None, order=None, place=None), Y=None, out=None) == aser.ASER_OK


def test_workspace_sizes():
    lib = aser.load_library()
    tail = lib.aser_mx4_forward_workspace_bytes(100, 256, 64, 0)
    assert tail == 256 and lib.aser_route_workspace_bytes(32, 64, 4) == tail and lib.aser_expert_forward_workspace_bytes(0, 256, 64, 4, 8) == tail
    assert lib.aser_mx4_forward_workspace_bytes(100, 256, 64, 8) > tail and lib.aser_route_workspace_bytes(33, 64, 4) >= tail + 2 * 64 * 4
    # many rows of experts are put in order: a place for each position
    for experts in (8, 1):
        assert lib.aser_expert_forward_workspace_bytes(100000, 256, 4096, experts, 0) >= tail + 100000 * 2 * 68
    assert lib.aser_mx4_forward_workspace_bytes(100000, 256, 4096, 0) == tail


# ------------------------------------------------------------------------------------------------ what the binding refuses
torch = pytest.importorskip("torch")
U8, I32 = torch.uint8, torch.int32


class Library:
    """Takes every call, remembers its name and returns ASER_OK."""

    def __init__(self):
        self.calls = []

    def __getattr__(self, name):
        def call(*args):
            self.calls.append(name)
            return aser.ASER_OK
        return call


@pytest.fixture
def stub():
    c = aser.Context.__new__(aser.Context)
    c._lib, c.handle, c.device, c._ws, c._ws_bytes = Library(), 1, torch.zeros(1).get_device(), None, 0
    return c


def zeros(*shape, dtype=torch.float32):
    return torch.zeros(*shape, dtype=dtype)


def tensors(rows=20, n=300, count=None):
    front = () if count is None else (count,)
    return zeros(*front, (rows + 15) // 16, 3, 4, 16, 16, dtype=U8), zeros(*front, (rows + 15) // 16, 3, 16, 4, dtype=U8)


def own_plan(rows=20, k=2, experts=4, **kw):
    a = dict(ids=zeros(rows, k, dtype=I32), weights=zeros(rows, k), offsets=zeros(experts + 1, dtype=I32), order=zeros(rows * k, dtype=I32), place=zeros(rows * k, dtype=I32))
    a.update(kw)
    return aser.ExpertPlan(**a)


def test_rows_side_by_side_are_laid_out():
    codes = torch.randint(0, 256, (2, 37, 192), dtype=U8)
    scales = torch.randint(0, 256, (2, 3, 37, 4), dtype=U8)
    m = aser.Mx4(codes, scales, 300)
    assert m.rows == 37 and m.count == 2 and tuple(m.codes.shape) == (2, 3, 3, 4, 16, 16) and tuple(m.scales.shape) == (2, 3, 3, 16, 4)
    for e, row, word, block in ((0, 0, 0, 0), (1, 17, 2, 3), (1, 36, 1, 1), (0, 15, 2, 0)):
        assert torch.equal(m.codes[e, row // 16, word, block, row % 16], codes[e, row, 64 * word + 16 * block:][:16])
        assert torch.equal(m.scales[e, row // 16, word, row % 16], scales[e, word, row])
    one = aser.Mx4(codes[0], scales[0], 300)
    assert torch.equal(one.codes, m.codes[0]) and one.count == 1


@pytest.mark.parametrize("make,error", [
    (lambda: aser.Mx4(*tensors(), 300), ValueError), (lambda: aser.Mx4(*tensors(), 400, 20), ValueError), (lambda: aser.Mx4(*tensors(), 300, 33), ValueError),
    (lambda: aser.Mx4(tensors()[0].to(torch.int8), tensors()[1], 300, 20), TypeError), (lambda: aser.Mx4(tensors()[0].transpose(0, 1).contiguous().transpose(0, 1), tensors()[1], 300, 20), ValueError),
    (lambda: aser.Mx4(zeros(20, 192, dtype=U8), zeros(3, 21, 4, dtype=U8), 300), ValueError), (lambda: own_plan(weights=zeros(20, 3)), ValueError),
    (lambda: own_plan(order=zeros(39, dtype=I32)), ValueError), (lambda: own_plan(ids=zeros(20, 2, dtype=torch.int64)), TypeError),
    (lambda: own_plan(weights=zeros(20, 2, dtype=torch.float64)), TypeError), (lambda: own_plan(ids=zeros(2, 20, dtype=I32).t()), ValueError)])
def test_holders_refuse(make, error):
    with pytest.raises(error):
        make()


def test_binding_refuses(stub):
    bf16 = torch.bfloat16
    x, w, ws = aser.Mx4(*tensors(), 300, 20), aser.Mx4(*tensors(48), 300, 48), aser.Mx4(*tensors(48, count=4), 300, 48)
    a, b = zeros(48, 8, dtype=bf16), zeros(8, 300, dtype=bf16)
    y, big = zeros(20, 48), zeros(40, 48)
    bad = [
        (ValueError, lambda: aser.aser_mx4_quantize(stub, zeros(19, 300), x)), (ValueError, lambda: aser.aser_mx4_quantize(stub, zeros(20, 299), x)),
        (TypeError, lambda: aser.aser_mx4_quantize(stub, zeros(20, 300, dtype=torch.float64), x)), (ValueError, lambda: aser.aser_mx4_quantize(stub, zeros(20, 300), x, mdiag=zeros(299))),
        (TypeError, lambda: aser.aser_mx4_quantize(stub, zeros(20, 300), x, mdiag=zeros(300, dtype=bf16))),
        (TypeError, lambda: aser.aser_mx4_quantize(stub, zeros(20, 300), x, values=zeros(20, 300, dtype=bf16))),
        (ValueError, lambda: aser.aser_mx4_quantize(stub, zeros(20, 300), x, values=zeros(20, 256))),
        (ValueError, lambda: aser.aser_mx4_forward(stub, x, w, zeros(19, 48))), (ValueError, lambda: aser.aser_mx4_forward(stub, x, w, zeros(20, 47))),
        (TypeError, lambda: aser.aser_mx4_forward(stub, x, w, zeros(20, 48, dtype=torch.float16))), (ValueError, lambda: aser.aser_mx4_forward(stub, x, w, y, L_A=a)),
        (ValueError, lambda: aser.aser_mx4_forward(stub, x, w, y, L_A=a[:47], L_B=b)), (ValueError, lambda: aser.aser_mx4_forward(stub, x, w, y, L_A=a, L_B=b[:, :256])),
        (TypeError, lambda: aser.aser_mx4_forward(stub, x, w, y, L_A=a.float(), L_B=b)), (ValueError, lambda: aser.aser_mx4_forward(stub, x, w, y, L_A=a[None], L_B=b[None])),
        (ValueError, lambda: aser.aser_route_experts(stub, zeros(20, 5), own_plan())), (ValueError, lambda: aser.aser_route_experts(stub, zeros(19, 4), own_plan())),
        (ValueError, lambda: aser.aser_route_experts(stub, zeros(20, 4), own_plan(), bias=zeros(3))), (TypeError, lambda: aser.aser_route_experts(stub, zeros(20, 4), own_plan(), bias=zeros(4, dtype=bf16))),
        (ValueError, lambda: aser.aser_expert_forward(stub, x, ws, own_plan(), zeros(39, 48), gather=True)),
        (ValueError, lambda: aser.aser_expert_forward(stub, x, ws, own_plan(), big, gather=True, L_A=a, L_B=b)),
        (ValueError, lambda: aser.aser_expert_combine(stub, zeros(39, 48), own_plan(), y)), (ValueError, lambda: aser.aser_expert_combine(stub, big, own_plan(), zeros(20, 47))),
        (TypeError, lambda: aser.aser_expert_combine(stub, big, own_plan(), y, Y0=zeros(20, 48, dtype=bf16))),
    ]
    for i, (error, call) in enumerate(bad):
        with pytest.raises(error):
            call()
        assert not stub._lib.calls, i
    stub.device = 3                                                              # tensors of another device than the context's
    for call in (lambda: aser.aser_mx4_quantize(stub, zeros(20, 300), x), lambda: aser.aser_mx4_forward(stub, x, w, y), lambda: aser.aser_route_experts(stub, zeros(20, 4), own_plan()),
                 lambda: aser.aser_expert_forward(stub, x, ws, own_plan(), big, gather=True), lambda: aser.aser_expert_combine(stub, big, own_plan(), y)):
        with pytest.raises(ValueError):
            call()
    assert not stub._lib.calls
    stub.device = torch.zeros(1).get_device()
    aser.aser_mx4_quantize(stub, zeros(20, 300), x, mdiag=zeros(300), values=zeros(20, 304)[:, :300])
    aser.aser_mx4_forward(stub, x, w, zeros(20, 24), swiglu=True, L_A=a, L_B=b)
    aser.aser_route_experts(stub, zeros(20, 4, dtype=bf16), own_plan(), bias=zeros(4))
    aser.aser_expert_forward(stub, x, ws, own_plan(), big, gather=True)
    aser.aser_expert_combine(stub, big, own_plan(), y, Y0=y)
    assert len(stub._lib.calls) == 5


@pytest.mark.parametrize("end", ["middle", "small", "large"])
def test_inputs_for_ranks_tell_terms_apart(end):
    """What the tests of P on the device would see of a P held as one, two or three terms: with the tolerances of fp32 outputs fewer than three fail, with those of
    bf16 outputs fewer than two, and at the ends of the range any number does."""
    import numpy as np

    import mx4_ranks
    _, _, L_A, _, P, Z, S = mx4_ranks.ranks_alone(np.random.default_rng(3), 300, 256, 400, 40, end)
    there = np.isfinite(Z)
    assert there.all(1).sum() == 299 and np.array_equal(P[:-1].astype(np.float32).astype(np.float64), P[:-1])
    for bf16, enough in ((False, 3), (True, 2)):
        for count in (1, 2, 3):
            with np.errstate(all="ignore"):
                held = np.abs(mx4_ranks.terms(P, count) @ L_A.T - Z) <= mx4_ranks.off(S, Z, bf16, True, False)
            assert held[there].all() == (count >= enough and end == "middle"), (bf16, count)


@pytest.mark.parametrize("n,m,r,experts", [(4096, 512, 64, 1), (4096, 1024, 64, 64), (4096, 14336, 32, 8), (1000, 48, 128, 1), (300, 6000, 1, 3), (128, 64, 16, 1024), (8192, 2048, 0, 16)])
def test_workspace_for_the_largest_batch_is_enough_for_the_others(n, m, r, experts):
    """A caller who asks for the largest number of rows has what every smaller one needs."""
    lib = aser.load_library()
    rows = list(range(1, 5000)) + [5000 + 37 * i for i in range(1500)]
    for need in ([lib.aser_mx4_forward_workspace_bytes(t, n, m, r) for t in rows], [lib.aser_expert_forward_workspace_bytes(t, n, m, experts, r) for t in rows],
                 [lib.aser_route_workspace_bytes(t, experts, 1) for t in rows]):
        falls = [(t, b - a) for t, a, b in zip(rows[1:], need, need[1:]) if b < a]
        assert not falls, falls[:3]


def test_forward_refuses_more_threads_than_a_launch_takes(ctx):
    most = (1 << 26) - 1                                                         # 2^21 tiles of 32 rows
    assert forward(ctx, x=mx(most), r=128, a=P, b=P) == SHAPE and "too many rows" in ctx.last_error()
    assert forward(ctx, x=mx(most), r=96, a=P, b=P) == ROOM
