"""Host-side checks of the serving entry points: what they refuse, before any HIP call is made."""
import ctypes

import pytest

import paper_2411_07762_amd as aser

P = 0x7F0000001000  # a fake, aligned "device address": validation must fail before it is touched


@pytest.fixture(scope="module")
def ctx():
    lib = aser.load_library()
    h = ctypes.c_void_p()
    assert lib.aser_create(ctypes.byref(h), 0, None) == aser.ASER_OK
    c = aser.Context.__new__(aser.Context)
    c._lib, c.handle, c.device, c._ws, c._ws_bytes = lib, h, 0, None, 0
    yield c
    c.close()


def cache(**kw):
    c = aser.aser_kv_cache(P, P, None, None, 100, 8 * 32 * 128, 32 * 128, 128, aser.ASER_KV_BF16, 32, 8, 128)
    for k, v in kw.items():
        setattr(c, k, v)
    return ctypes.byref(c)


def batch(**kw):
    b = aser.aser_kv_batch(P, P, P, 40, 4, 4, 1, 1000)
    for k, v in kw.items():
        setattr(b, k, v)
    return ctypes.byref(b)


BAD_CACHE = [
    (dict(k=None), aser.ASER_ERR_INVALID_ARG), (dict(v=None), aser.ASER_ERR_INVALID_ARG), (dict(k=P + 8), aser.ASER_ERR_INVALID_ARG),
    (dict(dtype=2), aser.ASER_ERR_DTYPE), (dict(dtype=aser.ASER_KV_INT8), aser.ASER_ERR_INVALID_ARG),
    (dict(dtype=aser.ASER_KV_INT8, k_scale=P, v_scale=P + 4), aser.ASER_ERR_INVALID_ARG),
    (dict(page_size=0), aser.ASER_ERR_SHAPE), (dict(page_size=8), aser.ASER_ERR_SHAPE), (dict(page_size=48), aser.ASER_ERR_SHAPE),
    (dict(page_size=512), aser.ASER_ERR_SHAPE), (dict(head_dim=96), aser.ASER_ERR_SHAPE), (dict(n_kv=0), aser.ASER_ERR_SHAPE),
    (dict(n_kv=5), aser.ASER_ERR_SHAPE), (dict(n_pages=0), aser.ASER_ERR_SHAPE), (dict(n_pages=1 << 31), aser.ASER_ERR_SHAPE),
    (dict(slot_stride=120), aser.ASER_ERR_SHAPE), (dict(slot_stride=136), aser.ASER_ERR_SHAPE), (dict(head_stride=-16), aser.ASER_ERR_SHAPE),
    (dict(page_stride=8), aser.ASER_ERR_SHAPE),
]
BAD_BATCH = [
    (dict(start=None), aser.ASER_ERR_INVALID_ARG), (dict(kv_len=None), aser.ASER_ERR_INVALID_ARG), (dict(pages=None), aser.ASER_ERR_INVALID_ARG),
    (dict(start=P + 2), aser.ASER_ERR_INVALID_ARG), (dict(n_seq=0), aser.ASER_ERR_SHAPE), (dict(n_seq=70000), aser.ASER_ERR_SHAPE),
    (dict(tokens=-1), aser.ASER_ERR_SHAPE), (dict(max_new=-1), aser.ASER_ERR_SHAPE), (dict(max_kv=-1), aser.ASER_ERR_SHAPE),
    (dict(max_kv=1281), aser.ASER_ERR_SHAPE), (dict(ld_pages=31), aser.ASER_ERR_SHAPE),
]


def attention(ctx, c, b, q=P, ldq=4096, heads=32, scale=0.1, window=0, sinks=0, out=P, ldo=4096):
    return ctx._lib.aser_paged_attention(ctx.handle, q, ldq, heads, c, b, scale, window, sinks, out, ldo)


def append(ctx, c, b, q=P, ldq=4096, heads=32, k=P, ldk=1024, v=P, ldv=1024, dt=0, opts=None, q_out=P, ldqo=4096):
    return ctx._lib.aser_kv_append(ctx.handle, q, ldq, heads, k, ldk, v, ldv, dt, ctypes.byref(opts) if opts else None, c, b, q_out, ldqo)


@pytest.mark.parametrize("call", [attention, append], ids=["attention", "append"])
def test_cache_and_batch_are_checked(ctx, call):
    for kw, status in BAD_CACHE:
        assert call(ctx, cache(**kw), batch()) == status, kw
    for kw, status in BAD_BATCH:
        assert call(ctx, cache(), batch(**kw)) == status, kw
    assert call(ctx, None, batch()) == aser.ASER_ERR_INVALID_ARG
    assert call(ctx, cache(), None) == aser.ASER_ERR_INVALID_ARG
    assert "head_dim" in ctx.last_error() or "null" in ctx.last_error()


def test_attention_is_checked(ctx):
    for kw, status in [(dict(q=None), 1), (dict(out=None), 1), (dict(heads=30), 2), (dict(heads=0), 2), (dict(ldq=4088), 2), (dict(ldo=4095), 2),
                       (dict(ldq=4100), 1), (dict(q=P + 2), 1), (dict(window=-1), 2), (dict(sinks=-1), 2), (dict(scale=float("nan")), 1),
                       (dict(scale=float("inf")), 1)]:
        assert attention(ctx, cache(), batch(), **kw) == status, kw
    assert ctx._lib.aser_paged_attention(None, P, 4096, 32, cache(), batch(), 0.1, 0, 0, P, 4096) == aser.ASER_ERR_INVALID_ARG
    # one request with a long cache is split and joined: that takes workspace
    assert attention(ctx, cache(), batch(n_seq=1, tokens=1, max_kv=100000, ld_pages=4000)) == aser.ASER_ERR_WORKSPACE
    assert attention(ctx, cache(), batch(tokens=0)) == aser.ASER_OK


def test_append_is_checked(ctx):
    for kw, status in [(dict(k=None), 1), (dict(v=None), 1), (dict(q_out=None), 1), (dict(q=None), 1), (dict(dt=2), 3), (dict(heads=30), 2),
                       (dict(ldq=4088), 2), (dict(ldk=1016), 2), (dict(ldv=1000), 2), (dict(ldqo=4000), 2), (dict(ldk=1028), 1), (dict(v=P + 4), 1)]:
        assert append(ctx, cache(), batch(), **kw) == status, kw
    good = dict(rope_cos=P, rope_sin=P, n_pos=1000, rot_dim=128, eps=1e-6)
    for kw, status in [(dict(rope_sin=None), 1), (dict(rope_cos=P + 4), 1), (dict(q_norm=P + 4), 1), (dict(rot_dim=0), 2), (dict(rot_dim=136), 2),
                       (dict(rot_dim=24), 2), (dict(n_pos=999), 2), (dict(q_norm=P, eps=-1.0), 1), (dict(k_norm=P, eps=float("nan")), 1)]:
        assert append(ctx, cache(), batch(), opts=aser.aser_qk_opts(**{**good, **kw})) == status, kw
    assert append(ctx, cache(), batch(tokens=0)) == aser.ASER_OK


def test_adapters_are_checked(ctx):
    def call(X=P, dt=0, rows=4, n=64, ldx=64, ids=P, A=P, B=P, scale=None, na=3, r=8, m=32, Y0=P, ldy0=32, Y=P, ldy=32):
        return ctx._lib.aser_adapter_forward(ctx.handle, X, dt, rows, n, ldx, ids, A, B, scale, na, r, m, Y0, ldy0, Y, ldy)
    for kw, status in [(dict(X=None), 1), (dict(ids=None), 1), (dict(A=None), 1), (dict(B=None), 1), (dict(Y=None), 1), (dict(dt=5), 3), (dict(rows=-1), 2),
                       (dict(n=0), 2), (dict(m=0), 2), (dict(ldx=63), 2), (dict(ldy=31), 2), (dict(ldy0=31), 2), (dict(r=0), 2), (dict(r=129), 2),
                       (dict(na=0), 2), (dict(na=4097), 2), (dict(ids=P + 2), 1), (dict(X=P + 2, dt=1), 1), (dict(A=P + 1), 1), (dict(Y=P + 2, Y0=None), 1),
                       (dict(ldy=40), 2), (dict(scale=P + 2), 1)]:
        assert call(**kw) == status, kw
    assert call() == aser.ASER_ERR_WORKSPACE
    assert call(rows=0) == aser.ASER_OK


def test_workspace_queries():
    lib = aser.load_library()
    assert lib.aser_paged_attention_workspace_bytes(None, None, 8) == 256
    assert lib.aser_paged_attention_workspace_bytes(cache(), batch(n_seq=1, max_kv=100000), 32) > 256
    assert aser.aser_adapter_workspace_bytes(0, 8, 8, 8) == 256
    assert aser.aser_adapter_workspace_bytes(48, 4096, 4096, 16) >= 48 * 16 * 4


def test_matrices_without_rows_have_no_address(ctx):
    """A framework's matrix of no rows has a null pointer: still a no-op, and everything else is still checked."""
    assert attention(ctx, cache(), batch(tokens=0), q=None, out=None) == aser.ASER_OK
    assert append(ctx, cache(), batch(tokens=0), q=None, k=None, v=None, q_out=None) == aser.ASER_OK
    assert append(ctx, cache(), batch(tokens=0), k=None, v=None, q_out=None) == aser.ASER_OK
    assert attention(ctx, cache(head_dim=96), batch(tokens=0), q=None, out=None) == aser.ASER_ERR_SHAPE
    assert append(ctx, cache(), batch(tokens=0, start=None), q=None, k=None, v=None, q_out=None) == aser.ASER_ERR_INVALID_ARG
    assert attention(ctx, cache(), None, q=None, out=None) == aser.ASER_ERR_INVALID_ARG
    assert append(ctx, cache(), None, q=None, k=None, v=None, q_out=None) == aser.ASER_ERR_INVALID_ARG

    def adapters(rows, X=None, ids=None, A=P, Y=None, n=64):
        return ctx._lib.aser_adapter_forward(ctx.handle, X, 0, rows, n, 64, ids, A, P, None, 3, 8, 32, None, 32, Y, 32)
    assert adapters(0) == aser.ASER_OK
    assert adapters(0, A=None) == aser.ASER_ERR_INVALID_ARG and adapters(0, n=0) == aser.ASER_ERR_SHAPE
    assert adapters(1) == adapters(1, X=P) == adapters(1, X=P, ids=P) == adapters(1, ids=P, Y=P) == aser.ASER_ERR_INVALID_ARG
