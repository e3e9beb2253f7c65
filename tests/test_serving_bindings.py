"""What the Python binding of the serving operators refuses before it hands addresses to the library: a stub stands for the library,
so that a call that is let through is seen and nothing runs."""
import pytest
import torch

import paper_2411_07762_amd as aser


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
def ctx():
    c = aser.Context.__new__(aser.Context)
    c._lib, c.handle, c.device, c._ws, c._ws_bytes = Library(), 1, torch.zeros(1).get_device(), None, 0
    return c


def zeros(*shape, dtype=torch.float32):
    return torch.zeros(*shape, dtype=dtype)


TOKENS, HEADS, KV, D, PAGE = 6, 4, 2, 64, 16


def cache():
    return aser.KvCache(*(zeros(5, KV, PAGE, D, dtype=torch.bfloat16) for _ in range(2)))


def batch(columns=3, max_kv=40):
    ints = torch.int32
    return aser.KvBatch(zeros(3, dtype=ints), zeros(2, dtype=ints), zeros(2, columns, dtype=ints), tokens=TOKENS, max_new=4, max_kv=max_kv)


def append(ctx, **kw):
    a = dict(q=zeros(TOKENS, HEADS * D), k=zeros(TOKENS, KV * D), v=zeros(TOKENS, KV * D), out=zeros(TOKENS, HEADS * D, dtype=torch.bfloat16),
             rope_cos=zeros(64, D // 2), rope_sin=zeros(64, D // 2), q_norm=zeros(D), k_norm=zeros(D))
    a.update(kw)
    return aser.aser_kv_append(ctx, a.pop("q"), a.pop("k"), a.pop("v"), a.pop("cache", None) or cache(), a.pop("batch", None) or batch(), a.pop("out"), **a)


def refused(ctx, error, call, **kw):
    with pytest.raises(error):
        call(ctx, **kw)
    assert not ctx._lib.calls, "the library was called"


@pytest.mark.parametrize("kw,error", [
    (dict(q_norm=zeros(D, dtype=torch.bfloat16)), TypeError), (dict(k_norm=zeros(D, dtype=torch.float64)), TypeError),
    (dict(q_norm=zeros(3)), ValueError), (dict(k_norm=zeros(2 * D)), ValueError),
    (dict(k_norm=zeros(2 * D)[::2]), ValueError),
    (dict(rope_cos=zeros(64, D // 2, dtype=torch.bfloat16), rope_sin=zeros(64, D // 2, dtype=torch.bfloat16)), TypeError),
    (dict(rope_sin=zeros(64, D // 2, dtype=torch.bfloat16)), TypeError), (dict(rope_sin=None), ValueError),
    (dict(rope_cos=None, q_norm=None, k_norm=None), ValueError), (dict(rope_cos=None), ValueError), (dict(rope_sin=zeros(63, D // 2)), ValueError),
    (dict(rope_cos=zeros(64, D)[:, ::2]), ValueError),
])
def test_append_refuses_tables_and_weights_that_the_kernel_would_misread(ctx, kw, error):
    refused(ctx, error, append, **kw)
    assert append(ctx) == aser.ASER_OK and ctx._lib.calls == ["aser_kv_append"]
    assert append(ctx, rope_cos=None, rope_sin=None, q_norm=None, k_norm=zeros(1, D)) == aser.ASER_OK


def attention(ctx, **kw):
    a = dict(q=zeros(TOKENS, HEADS * D, dtype=torch.bfloat16), out=zeros(TOKENS, HEADS * D, dtype=torch.bfloat16))
    a.update(kw)
    return aser.aser_paged_attention(ctx, a["q"], a.get("cache") or cache(), a.get("batch") or batch(), a["out"], scale=0.1)


def test_heads_that_the_rows_do_not_have_are_refused(ctx):
    """A slice of fewer heads' columns than the cache has reads its neighbours', and past the last row."""
    fused = zeros(TOKENS, 3 * KV * D)
    for name in "kv":
        refused(ctx, ValueError, append, **{name: fused[:, :KV * D - D]})
        refused(ctx, ValueError, append, **{name: fused[:, :KV * D - 1]})
    refused(ctx, ValueError, append, q=zeros(TOKENS, HEADS * D + 8), out=zeros(TOKENS, HEADS * D + 8, dtype=torch.bfloat16))
    refused(ctx, ValueError, attention, q=zeros(TOKENS, HEADS * D - 16, dtype=torch.bfloat16))
    assert append(ctx, k=fused[:, :KV * D], v=fused[:, KV * D:2 * KV * D]) == aser.ASER_OK
    assert append(ctx, q=None, out=None) == aser.ASER_OK
    assert attention(ctx, q=zeros(TOKENS, D * KV, dtype=torch.bfloat16)) == aser.ASER_OK


def adapters(ctx, **kw):
    a = dict(X=zeros(TOKENS, 32), adapter=zeros(TOKENS, dtype=torch.int32), A=zeros(3, 4, 32, dtype=torch.bfloat16), B=zeros(3, 20, 4, dtype=torch.bfloat16),
             scale=zeros(3), Y0=None, Y=zeros(TOKENS, 20))
    a.update(kw)
    return aser.aser_adapter_forward(ctx, a["X"], a["adapter"], a["A"], a["B"], a["scale"], a["Y0"], a["Y"])


@pytest.mark.parametrize("kw,error", [
    (dict(adapter=zeros(TOKENS)), TypeError), (dict(adapter=zeros(TOKENS, dtype=torch.int64)), TypeError),
    (dict(adapter=zeros(2 * TOKENS, dtype=torch.int32)[::2]), ValueError), (dict(adapter=zeros(TOKENS + 1, dtype=torch.int32)), ValueError),
    (dict(adapter=zeros(1, dtype=torch.int32).expand(TOKENS)), ValueError),
    (dict(scale=zeros(3, dtype=torch.bfloat16)), TypeError), (dict(scale=zeros(3, dtype=torch.float64)), TypeError),
    (dict(scale=zeros(2)), ValueError), (dict(scale=zeros(6)[::2]), ValueError), (dict(scale=zeros(1).expand(3)), ValueError),
])
def test_adapters_refuse_numbers_and_scales_that_the_kernel_would_misread(ctx, kw, error):
    refused(ctx, error, adapters, **kw)
    assert adapters(ctx) == aser.ASER_OK and adapters(ctx, scale=None) == aser.ASER_OK and adapters(ctx, scale=zeros(4)) == aser.ASER_OK
    assert adapters(ctx, X=zeros(1, 32), adapter=zeros(TOKENS, dtype=torch.int32)[:1], Y=zeros(1, 20)) == aser.ASER_OK


@pytest.mark.parametrize("call", [append, attention], ids=["append", "attention"])
def test_page_table_has_a_column_for_every_page(ctx, call):
    """A slice of columns has the wider table's leading dimension: its own are what counts."""
    table = zeros(2, 8, dtype=torch.int32)

    def of(pages, max_kv=40):
        return aser.KvBatch(zeros(3, dtype=torch.int32), zeros(2, dtype=torch.int32), pages, tokens=TOKENS, max_new=4, max_kv=max_kv)

    refused(ctx, ValueError, call, batch=of(table[:, :2]))
    refused(ctx, ValueError, call, batch=of(table[:, 6:]))
    refused(ctx, ValueError, call, batch=of(zeros(2, 3, dtype=torch.int32), 49))
    assert call(ctx, batch=of(table[:, :3])) == aser.ASER_OK and call(ctx, batch=of(table[:, 5:], 48)) == aser.ASER_OK


class There(torch.Tensor):
    """A tensor that says it is on device 3."""

    def get_device(self):
        return 3


def there(*shape, dtype=torch.float32):
    return torch.zeros(*shape, dtype=dtype).as_subclass(There)


def test_tensors_of_another_device_than_the_context_are_refused(ctx):
    """The address of a host tensor, or of another device's, would fault in the kernel."""
    ints, half, rows = torch.int32, torch.bfloat16, (TOKENS, HEADS * D)
    args = {append: dict(q=(rows,), k=((TOKENS, KV * D),), v=((TOKENS, KV * D),), out=(rows, half), rope_cos=((64, D // 2),), rope_sin=((64, D // 2),), q_norm=((D,),), k_norm=((D,),)),
            attention: dict(q=(rows, half), out=(rows, half)),
            adapters: dict(X=((TOKENS, 32),), adapter=((TOKENS,), ints), A=((3, 4, 32), half), B=((3, 20, 4), half), scale=((3,),), Y=((TOKENS, 20),), Y0=((TOKENS, 20),))}
    for call, names in args.items():
        for name, (shape, *dtype) in names.items():
            refused(ctx, ValueError, call, **{name: there(*shape, **dict(zip(["dtype"], dtype)))})
    pages = (5, KV, PAGE, D)
    with pytest.raises(ValueError):
        aser.KvCache(zeros(*pages, dtype=half), there(*pages, dtype=half))
    for at in range(2):
        scales = [zeros(*pages[:3]), zeros(*pages[:3])]
        scales[at] = there(*pages[:3])
        with pytest.raises(ValueError):
            aser.KvCache(zeros(*pages, dtype=torch.int8), zeros(*pages, dtype=torch.int8), *scales)
    for at in range(3):
        parts = [zeros(3, dtype=ints), zeros(2, dtype=ints), zeros(2, 3, dtype=ints)]
        parts[at] = there(*parts[at].shape, dtype=ints)
        with pytest.raises(ValueError):
            aser.KvBatch(*parts, tokens=TOKENS, max_new=4, max_kv=40)
    cache_there = aser.KvCache(there(*pages, dtype=half), there(*pages, dtype=half))
    batch_there = aser.KvBatch(there(3, dtype=ints), there(2, dtype=ints), there(2, 3, dtype=ints), tokens=TOKENS, max_new=4, max_kv=40)
    for call in (append, attention):
        refused(ctx, ValueError, call, cache=cache_there)
        refused(ctx, ValueError, call, batch=batch_there)
    ctx.device = 0                                        # everything else on the host
    for call in (append, attention, adapters):
        refused(ctx, ValueError, call)
