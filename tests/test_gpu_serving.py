"""The serving operators (cache append, paged attention, adapters) against the oracle in 64 bits.

Tolerances, element by element, from the formats: bf16 rounds by at most 2^-8 of the value.  Append: one such rounding, on
top of fp32 arithmetic on values of the row's size (2e-6 of its largest).  8-bit cache: half a step.  Attention: the output's
rounding, the probabilities' (2^-8 of sum p |v|) and 1e-4 of that sum for logits in fp32 (sums of up to 256 products: 1e-5 in a
logit) and the exponential.  Adapters: fp32 sums of n / 32 + r / 32 matrix instructions of 32 terms each, taken as 2^-23 a
step and 64 steps for everything around, of the sum of absolute terms.
"""
import numpy as np
import pytest
import torch

import paper_2411_07762_amd as aser
from oracle import serving_oracle as orc

from gpu_util import DEV, new_ctx
from test_gpu_parity import say

pytestmark = pytest.mark.gpu

BF16 = 2.0 ** -8


def f64(t):
    return t.detach().float().cpu().numpy().astype(np.float64)


class Requests:
    """Requests with new[s] new tokens and kv[s] cached ones, on shuffled pages; unused table entries are -1."""

    def __init__(self, new, kv, page, seed=1, spare=2, gap=0):
        rng = np.random.default_rng(seed)
        self.new, self.kv, self.page = list(new), list(kv), page
        per = [-(-n // page) for n in kv]
        self.n_pages = sum(per) + spare
        order = rng.permutation(self.n_pages)[:sum(per)]
        width = max(max(per), 1) + 1
        self.pages = np.full((len(kv), width), -1, np.int32)
        at = 0
        for s, c in enumerate(per):
            self.pages[s, :c] = order[at:at + c]
            at += c
        self.start = (gap + np.concatenate([[0], np.cumsum(new)])).astype(np.int32)
        self.tokens = int(self.start[-1]) + gap
        self.kv_len = np.array(kv, np.int32)

    def batch(self, **kw):
        dev = [torch.from_numpy(a).to(DEV) for a in (self.start, self.kv_len, self.pages)]
        bounds = dict(tokens=self.tokens, max_new=max(self.new), max_kv=max(self.kv))
        bounds.update(kw)
        return aser.KvBatch(*dev, **bounds)


def make_cache(req, kv_heads, d, int8, seed, slot_pad=0, slots_first=False):
    """A cache of random values; with slots_first the slots of a page come before its heads in memory."""
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    shape = (req.n_pages, kv_heads, req.page, d)
    mem = (req.n_pages, req.page, kv_heads, d + slot_pad) if slots_first else (req.n_pages, kv_heads, req.page, d + slot_pad)

    def one():
        if int8:
            t = torch.randint(-127, 128, mem, generator=g, device=DEV, dtype=torch.int8)
        else:
            t = torch.randn(mem, generator=g, device=DEV).to(torch.bfloat16)
        return (t.transpose(1, 2) if slots_first else t)[..., :d]

    scales = [(torch.rand(shape[:3], generator=g, device=DEV) + 0.5) / 73.0 for _ in range(2)] if int8 else [None, None]
    return aser.KvCache(one(), one(), *scales)


def numbers(cache):
    k, v = f64(cache.k), f64(cache.v)
    if cache.k_scale is not None:
        k, v = k * f64(cache.k_scale)[..., None], v * f64(cache.v_scale)[..., None]
    return k, v


# ------------------------------------------------------------------------------------------------ attention
def attend(req, cache, heads, scale=None, window=0, sinks=0, seed=3, q_scale=1.5, pad=0, ctx=None, **bounds):
    d = cache.c.head_dim
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    q = (q_scale * torch.randn(req.tokens, heads * d + pad, generator=g, device=DEV)).to(torch.bfloat16)[:, :heads * d]
    out = torch.full((req.tokens, heads * d + pad), 7.0, dtype=torch.bfloat16, device=DEV)
    ctx = ctx or new_ctx()
    batch = req.batch(**bounds)
    ctx.ensure_workspace(aser.aser_paged_attention_workspace_bytes(cache, batch, heads))
    scale = d ** -0.5 if scale is None else scale
    ctx.check(aser.aser_paged_attention(ctx, q, cache, batch, out[:, :heads * d], scale=scale, window=window, sinks=sinks))
    torch.cuda.synchronize()
    if pad:
        assert (out[:, heads * d:] == 7.0).all()
    return q, out[:, :heads * d]


def check_attention(label, req, cache, heads, q, out, scale=None, window=0, sinks=0, n_pages=None):
    d = cache.c.head_dim
    k, v = numbers(cache)
    scale = d ** -0.5 if scale is None else scale
    want, size = orc.attention(f64(q).reshape(req.tokens, heads, d), k, v, req.pages, req.start, req.kv_len, scale, window, sinks, n_pages)
    rows = slice(int(req.start[0]), int(req.start[-1]))
    got = f64(out).reshape(req.tokens, heads, d)
    outside = np.ones(req.tokens, bool)
    outside[rows] = False
    assert (got[outside] == 7.0).all(), "rows of no request were written"
    got, want, size = got[rows], want[rows], size[rows]
    assert np.isfinite(got).all()
    err, bar = np.abs(got - want), BF16 * np.abs(want) + (BF16 + 1e-4) * size
    rel = np.linalg.norm(got - want) / max(np.linalg.norm(want), 1e-30)
    say("%s: largest error / bound %.2f, relative %.2e" % (label, (err / np.maximum(bar, 1e-30)).max(), rel))
    assert (err <= bar).all()
    assert rel <= 3e-3


ATTENTION = [
    # new, kv, heads, kv_heads, d, page, int8, window, sinks
    ("one_key", [1], [1], 4, 4, 64, 16, False, 0, 0),
    ("one_token", [1], [77], 32, 8, 128, 64, False, 0, 0),
    ("page_ends_inside_a_tile", [1, 1, 1], [16, 17, 48], 8, 2, 128, 16, False, 0, 0),
    ("long_axis", [1], [5003], 16, 4, 128, 32, False, 0, 0),
    ("long_axis_256", [1, 1], [2049, 3], 8, 2, 256, 64, False, 0, 0),
    ("long_axis_int8", [1, 1], [4097, 1300], 8, 1, 64, 16, True, 0, 0),
    ("int8_128", [1] * 5, [31, 32, 33, 64, 700], 16, 4, 128, 128, True, 0, 0),
    ("int8_256", [2, 1], [130, 65], 4, 4, 256, 32, True, 0, 0),
    ("group_of_all_heads", [1, 1], [300, 299], 40, 1, 64, 32, False, 0, 0),
    ("group_of_three", [3, 1], [100, 40], 12, 4, 128, 16, False, 0, 0),
    ("several_tokens", [4, 1, 7, 2], [60, 1, 7, 900], 8, 8, 128, 32, False, 0, 0),
    ("request_without_tokens", [1, 0, 2], [50, 20, 2], 8, 2, 64, 16, False, 0, 0),
    ("window", [1, 1, 1], [10, 200, 5000], 8, 2, 128, 32, False, 100, 0),
    ("window_sinks", [1, 3, 1], [7, 500, 4001], 8, 2, 128, 32, False, 64, 4),
    ("window_of_one", [1, 5], [333, 40], 8, 2, 64, 16, False, 1, 0),
    ("sinks_beyond_window", [1, 9], [333, 80], 8, 2, 64, 16, True, 8, 200),
    ("prompt", [333], [333], 8, 2, 128, 64, False, 0, 0),
    ("prompt_64", [257, 1, 70], [257, 90, 300], 8, 8, 64, 16, False, 0, 0),
    ("prompt_256", [150, 20], [170, 20], 4, 1, 256, 32, False, 0, 0),
    ("prompt_behind_others", [130, 64], [1000, 64], 8, 1, 128, 256, False, 0, 0),
    ("prompt_int8", [200, 31], [300, 31], 8, 2, 128, 32, True, 0, 0),
    ("prompt_int8_64", [129, 300], [129, 2000], 8, 4, 64, 16, True, 0, 0),
    ("prompt_int8_256", [129], [200], 4, 2, 256, 16, True, 0, 0),
    ("prompt_window", [700, 40], [700, 400], 8, 2, 128, 32, False, 90, 0),
    ("prompt_window_sinks", [515, 129], [515, 1200], 4, 4, 64, 16, False, 64, 5),
    ("prompt_window_sinks_int8", [600], [777], 12, 4, 128, 64, True, 33, 40),
    ("prompt_group_of_five", [97, 261], [97, 300], 10, 2, 128, 32, False, 0, 0),
    ("prompt_group_of_all", [120], [121], 64, 1, 64, 32, False, 0, 0),
    ("prompt_long", [2100], [2100], 2, 1, 128, 128, False, 0, 0),
]


@pytest.mark.parametrize("name,new,kv,heads,kv_heads,d,page,int8,window,sinks", ATTENTION, ids=[c[0] for c in ATTENTION])
def test_attention(name, new, kv, heads, kv_heads, d, page, int8, window, sinks):
    say("attention case %s" % name)
    req = Requests(new, kv, page)
    cache = make_cache(req, kv_heads, d, int8, 5)
    q, out = attend(req, cache, heads, window=window, sinks=sinks)
    check_attention(name, req, cache, heads, q, out, window=window, sinks=sinks)


@pytest.mark.parametrize("int8", [False, True], ids=["bf16", "int8"])
@pytest.mark.parametrize("new", [[2, 1, 3], [150, 1, 40]], ids=["few", "prompt"])
def test_attention_strides_padding_and_rows_of_no_request(new, int8):
    """Slots before heads in memory, padded slots, padded rows of q and out, rows in front of and behind the requests'; max_new and
    max_kv above what is there."""
    say("attention strides %s int8=%s" % (new, int8))
    req = Requests(new, [300, 90, 161], 32, gap=2)
    cache = make_cache(req, 2, 128, int8, 6, slot_pad=16, slots_first=True)
    q, out = attend(req, cache, 8, pad=8, max_new=max(new) + 9, max_kv=320)
    check_attention("strides", req, cache, 8, q, out)


@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("new", [[1, 2], [100, 37]], ids=["few", "prompt"])
def test_attention_ignores_what_nobody_sees(new, d):
    """NaN and infinities in slots past the request's tokens, in keys that left the window and in pages that the table does not
    name; table entries outside [0, n_pages) hide their tokens."""
    say("attention unseen values %s d=%d" % (new, d))
    req = Requests(new, [200, 45], 16, spare=3)
    cache = make_cache(req, 2, d, False, 7)
    used = np.zeros((req.n_pages, req.page), bool)
    window = 48
    for s in range(2):
        low = req.kv[s] - new[s] - window + 1
        for p in range(req.kv[s]):
            used[req.pages[s, p // 16], p % 16] = p >= low or p < 4
    hide = torch.from_numpy(~used).to(DEV)[:, None, :, None]
    for t in (cache.k, cache.v):
        t.masked_fill_(hide, float("nan"))
    cache.v[hide.expand_as(cache.v) & (torch.arange(d, device=DEV) % 3 == 1)] = float("inf")
    q, out = attend(req, cache, 8, window=window, sinks=4)
    check_attention("unseen", req, cache, 8, q, out, window=window, sinks=4)
    # without a window: pages that are not there, in the middle, at the end, everywhere
    req = Requests(new, [200, 45], 16, seed=2)
    cache = make_cache(req, 2, d, False, 8)
    for at, bad in ((3, -1), (5, req.n_pages), (7, 2 ** 31 - 1), (12, -2 ** 31)):
        req.pages[0, at] = bad
    req.pages[1, :] = -7
    q, out = attend(req, cache, 8)
    check_attention("missing pages", req, cache, 8, q, out)
    assert (out[int(req.start[1]):int(req.start[2])] == 0).all()


def test_attention_clamps_what_the_device_says():
    """Lengths above max_kv, below zero, more new tokens than cached ones, starts outside the rows: nothing out of range is
    touched, tokens in front of position 0 see nothing."""
    say("attention clamps")
    req = Requests([2, 1, 3], [40, 33, 20], 16)
    cache = make_cache(req, 2, 64, False, 9)
    true = req.kv_len.copy()
    req.kv_len = np.array([1000, -5, 2], np.int32)
    q, out = attend(req, cache, 4, max_kv=40)
    req.kv_len = np.array([40, 0, 2], np.int32)
    got = f64(out)
    assert (got[2] == 0).all() and (got[3] == 0).all()
    k, v = numbers(cache)
    want, size = orc.attention(f64(q).reshape(6, 4, 64)[:2], k, v, req.pages[:1], req.start[:2], req.kv_len[:1], 64 ** -0.5)
    assert (np.abs(got[:2].reshape(2, 4, 64) - want) <= BF16 * np.abs(want) + (BF16 + 1e-4) * size).all()
    want, size = orc.attention(f64(q).reshape(6, 4, 64)[4:], k, v, req.pages[2:], np.array([0, 2]), np.array([2]), 64 ** -0.5)
    assert (np.abs(got[4:].reshape(2, 4, 64) - want) <= BF16 * np.abs(want) + (BF16 + 1e-4) * size).all()
    req.kv_len = true
    req.start = np.array([-3, 2, 900, 5], np.int32)      # request 1: rows 2 .. 5, request 2: none (the end comes first)
    _, out = attend(req, cache, 4, max_kv=40, max_new=6)
    assert np.isfinite(f64(out)).all()


def test_attention_logits_far_apart():
    """Logits of hundreds, rising along the axis (the maximum moves many times) and falling (it never does)."""
    say("attention far logits")
    for new in ([1], [70]):
        for sign in (1.0, -1.0):
            req = Requests(new, [1500], 32)
            cache = make_cache(req, 1, 128, False, 10)
            ramp = torch.linspace(-1, 1, req.n_pages * 32, device=DEV).reshape(-1)[:1500]
            for p in range(0, 1500, 32):
                n = min(32, 1500 - p)
                cache.k[req.pages[0, p // 32], 0, :n, :] = (sign * ramp[p:p + n, None]).to(torch.bfloat16)
            d = 128
            q = torch.ones(req.tokens, 4 * d, device=DEV).to(torch.bfloat16) * 3
            out = torch.empty_like(q)
            ctx, batch = new_ctx(), req.batch()
            ctx.ensure_workspace(aser.aser_paged_attention_workspace_bytes(cache, batch, 4))
            ctx.check(aser.aser_paged_attention(ctx, q, cache, batch, out, scale=1.0))
            torch.cuda.synchronize()
            check_attention("ramp %+.0f" % sign, req, cache, 4, q, out, scale=1.0)


def test_attention_page_offsets_beyond_32_bits():
    """Pages further than 2^31 elements into the cache."""
    say("attention long cache")
    stride = (1 << 31) // 40 // 16 * 16 + 16 * 1024
    buf = torch.zeros(48 * stride, dtype=torch.bfloat16, device=DEV)
    view = buf.as_strided((48, 2, 64, 64), (stride, 64 * 64, 64, 1))
    req = Requests([1, 30], [100, 130], 64)
    req.pages[0, :2], req.pages[1, :3] = [47, 1], [46, 45, 0]
    g = torch.Generator(device=DEV)
    g.manual_seed(1)
    kv = []
    for t in (view, buf[2 * 64 * 64:].as_strided((48, 2, 64, 64), (stride, 64 * 64, 64, 1))):
        for p in (47, 1, 46, 45, 0):
            t[p] = torch.randn(2, 64, 64, generator=g, device=DEV).to(torch.bfloat16)
        kv.append(t)
    cache = aser.KvCache(*kv)
    q, out = attend(req, cache, 4)
    check_attention("long cache", req, cache, 4, q, out)


def test_attention_repeats_and_follows_its_stream():
    """The same bits from call to call, also as a replayed graph on another stream with other work between the replays."""
    say("attention graph")
    req = Requests([1, 1, 40], [3000, 700, 41], 32)
    cache = make_cache(req, 2, 128, False, 11)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        ctx = new_ctx()
        q, first = attend(req, cache, 8, ctx=ctx)
        batch = req.batch()
        out = torch.zeros_like(first)
        graph = torch.cuda.CUDAGraph()
        side.synchronize()
        with torch.cuda.graph(graph, stream=side):
            ctx.check(aser.aser_paged_attention(ctx, q, cache, batch, out, scale=128 ** -0.5))
        for _ in range(4):
            out.zero_()
            graph.replay()
            torch.randn(1000, device=DEV).sum().item()
            assert torch.equal(out, first)



@pytest.mark.parametrize("kv_heads", [1, 2, 8])
@pytest.mark.parametrize("longest", [5, 12, 16, 40])
def test_attention_of_single_tokens_beside_longer_requests(longest, kv_heads):
    """Requests of one to four row tiles, and a prompt, in one call."""
    new = [1, longest, 1, 1, 3, 1, max(longest // 2, 1), 1, 0, 1, 4, 1]
    kv = [700, 90, 1, 333, 64, 2000, 150, 17, 40, 512, 31, 1025]
    req = Requests(new, kv, 32, seed=longest)
    heads = 4 * kv_heads
    cache = make_cache(req, kv_heads, 64, False, 21)
    q, out = attend(req, cache, heads)
    check_attention("single tokens beside %d, %d key/value heads" % (longest, kv_heads), req, cache, heads, q, out)


@pytest.mark.parametrize("int8", [False, True], ids=["bf16", "int8"])
@pytest.mark.parametrize("d", [64, 128, 256])
def test_attention_of_more_rows_than_the_device_holds_at_once(d, int8):
    """40 requests that are one and the same: each has the first one's result to the bit, however their workgroups follow one another."""
    new, kv, heads, kv_heads, copies = 260, 330, 32, 8, 40
    req = Requests([new], [kv], 32)
    cache = make_cache(req, kv_heads, d, int8, 11)
    q, out = attend(req, cache, heads)
    check_attention("one of %d, %d channels%s" % (copies, d, ", int8" if int8 else ""), req, cache, heads, q, out)
    many = Requests([new], [kv], 32)
    many.new, many.kv = [new] * copies, [kv] * copies
    many.pages = np.repeat(req.pages, copies, axis=0)
    many.start = (new * np.arange(copies + 1)).astype(np.int32)
    many.kv_len = np.full(copies, kv, np.int32)
    many.tokens = new * copies
    all_q = q.repeat(copies, 1)
    ctx, batch = new_ctx(), many.batch()
    ctx.ensure_workspace(aser.aser_paged_attention_workspace_bytes(cache, batch, heads))
    got = torch.empty(many.tokens, heads * d, dtype=torch.bfloat16, device=DEV)
    for _ in range(3):
        got.fill_(7.0)
        ctx.check(aser.aser_paged_attention(ctx, all_q, cache, batch, got, scale=d ** -0.5))
        torch.cuda.synchronize()
        views = got.view(copies, new, heads * d)
        wrong = [s for s in range(copies) if not torch.equal(views[s], views[0])]
        assert not wrong, "requests %s differ from the first" % wrong
        assert torch.equal(views[0], views[copies - 1])
        bar = BF16 * out.float().abs().max().item()
        assert (views[0].float() - out.float()).abs().max().item() <= 2 * bar


# ------------------------------------------------------------------------------------------------ append
APPEND = [
    # new, kv, heads, kv_heads, d, page, x, int8, norm, style, rot
    ("one_token", [1], [1], 4, 2, 64, 16, "f32", False, False, "half", 64),
    ("one_token_far", [1], [1000], 32, 8, 128, 64, "bf16", False, False, "half", 128),
    ("batch_norm", [1] * 70, [1 + 7 * i for i in range(70)], 8, 2, 128, 32, "bf16", False, True, "half", 128),
    ("prompts", [100, 0, 33, 1], [100, 5, 60, 1], 6, 3, 64, 16, "f32", False, True, "pairs", 64),
    ("half_rotated", [40, 3], [40, 90], 8, 1, 128, 128, "f32", False, False, "half", 64),
    ("quarter_rotated_pairs", [17], [30], 4, 4, 256, 32, "bf16", False, True, "pairs", 64),
    ("sixteen_rotated", [19], [30], 4, 4, 64, 32, "bf16", False, False, "half", 16),
    ("not_rotated", [9, 8], [9, 50], 4, 2, 128, 16, "f32", False, True, None, 0),
    ("int8", [70, 1, 2], [70, 200, 2], 8, 2, 128, 64, "f32", True, True, "half", 128),
    ("int8_64", [33, 1], [40, 17], 4, 4, 64, 16, "bf16", True, False, "pairs", 64),
    ("int8_256", [5], [300], 4, 1, 256, 256, "bf16", True, False, "half", 128),
    ("many_tokens", [5000], [5003], 8, 1, 64, 64, "bf16", False, True, "half", 64),
]


@pytest.mark.parametrize("name,new,kv,heads,kv_heads,d,page,x,int8,norm,style,rot", APPEND, ids=[c[0] for c in APPEND])
@pytest.mark.parametrize("fused", [False, True], ids=["apart", "fused"])
def test_append(name, new, kv, heads, kv_heads, d, page, x, int8, norm, style, rot, fused):
    say("append case %s fused=%s" % (name, fused))
    req = Requests(new, kv, page, gap=1)
    g = torch.Generator(device=DEV)
    g.manual_seed(4)
    T, dt = req.tokens, torch.float32 if x == "f32" else torch.bfloat16
    if fused:
        qkv = torch.randn(T, (heads + 2 * kv_heads) * d, generator=g, device=DEV).to(dt)
        q, k, v = qkv[:, :heads * d], qkv[:, heads * d:(heads + kv_heads) * d], qkv[:, (heads + kv_heads) * d:]
    else:
        q, k, v = (torch.randn(T, n * d, generator=g, device=DEV).to(dt) for n in (heads, kv_heads, kv_heads))
    v[T // 2] = 0
    cache = make_cache(req, kv_heads, d, int8, 12, slots_first=fused)
    before = [t.clone() for t in (cache.k, cache.v)] + [None if t is None else t.clone() for t in (cache.k_scale, cache.v_scale)]
    cos = sin = qn = kn = None
    if style:
        angle = torch.arange(max(kv) + 3, dtype=torch.float64, device=DEV)[:, None] * 10000.0 ** (-torch.arange(0, rot, 2, dtype=torch.float64, device=DEV) / rot)
        cos, sin = angle.cos().float(), angle.sin().float()
    if norm:
        qn, kn = (1 + 0.1 * torch.randn(d, generator=g, device=DEV) for _ in range(2))
    out = torch.full((T, heads * d), 7.0, dtype=torch.bfloat16, device=DEV)
    ctx = new_ctx()
    ctx.check(aser.aser_kv_append(ctx, q, k, v, cache, req.batch(), out, rope_cos=cos, rope_sin=sin, interleaved=style == "pairs", q_norm=qn, k_norm=kn))
    torch.cuda.synchronize()
    cos, sin, qn, kn = (None if t is None else t.cpu().numpy() for t in (cos, sin, qn, kn))
    want_q = np.full((T, heads, d), 7.0)
    written = np.zeros((req.n_pages, page), bool)
    kw, vw = np.zeros((req.n_pages, kv_heads, page, d)), np.zeros((req.n_pages, kv_heads, page, d))
    for s in range(len(new)):
        rows, pos = slice(req.start[s], req.start[s + 1]), orc.positions_of(req.start, req.kv_len, s)
        if not len(pos):
            continue
        shape = (len(pos), -1, d)
        want_q[rows] = orc.turned(f64(q)[rows].reshape(shape), pos, cos, sin, style == "pairs", qn, 1e-6)
        at, slot = req.pages[s][pos // page], pos % page
        written[at, slot] = True
        kw[at, :, slot] = orc.turned(f64(k)[rows].reshape(shape), pos, cos, sin, style == "pairs", kn, 1e-6)
        vw[at, :, slot] = f64(v)[rows].reshape(shape)
    got = f64(out).reshape(T, heads, d)
    assert (np.abs(got - want_q) <= BF16 * np.abs(want_q) + 2e-6 * np.abs(want_q).max(-1, keepdims=True)).all()
    for got, want, old, sc, sc_old in ((cache.k, kw, before[0], cache.k_scale, before[2]), (cache.v, vw, before[1], cache.v_scale, before[3])):
        w = np.broadcast_to(written[:, None], got.shape[:3])
        assert np.array_equal(f64(got)[~w], f64(old)[~w]), "other slots were written"
        top = np.abs(want).max(-1, keepdims=True)
        if int8:
            assert np.array_equal(f64(sc)[~w], f64(sc_old)[~w])
            scale = np.where(top == 0, 1.0, top / 127.0)
            assert (np.abs(f64(sc)[..., None] - scale)[w] <= 2e-6 * scale[w]).all()
            codes = f64(got)
            assert np.abs(codes).max() <= 127
            assert (np.abs(codes * f64(sc)[..., None] - want)[w] <= 0.5 * scale[w] + 3e-6 * top[w]).all()
        else:
            assert (np.abs(f64(got) - want)[w] <= (BF16 * np.abs(want) + 2e-6 * top)[w]).all()


def test_append_skips_what_is_not_there():
    """Pages that the table does not have, positions in front of 0, no queries."""
    say("append missing pages")
    req = Requests([20, 4], [40, 10], 16)
    req.pages[0, 2], req.pages[1, 0] = -1, req.n_pages
    req.kv_len[1] = 2                                      # two of four tokens lie in front of position 0
    g = torch.Generator(device=DEV)
    g.manual_seed(2)
    k, v, q = (torch.randn(24, n, generator=g, device=DEV) for n in (128, 128, 256))
    cache = make_cache(req, 2, 64, False, 13)
    old_k, old_v = cache.k.clone(), cache.v.clone()
    out = torch.full((24, 256), 7.0, dtype=torch.bfloat16, device=DEV)
    ctx = new_ctx()
    ctx.check(aser.aser_kv_append(ctx, q, k, v, cache, req.batch(), out))
    torch.cuda.synchronize()
    assert torch.equal(out[:20], q[:20].to(torch.bfloat16)) and (out[20:22] == 7).all() and torch.equal(out[22:], q[22:].to(torch.bfloat16))
    want_k, want_v = old_k, old_v
    for t in range(12):                                    # positions 20 .. 31 on page 1; 32 .. 39 are on the missing one
        want_k[req.pages[0, 1], :, 4 + t] = k[t].reshape(2, 64).to(torch.bfloat16)
        want_v[req.pages[0, 1], :, 4 + t] = v[t].reshape(2, 64).to(torch.bfloat16)
    assert torch.equal(cache.k, want_k) and torch.equal(cache.v, want_v)
    cache.k.zero_()
    ctx.check(aser.aser_kv_append(ctx, None, k, v, cache, req.batch(), None))
    torch.cuda.synchronize()
    assert torch.equal(cache.k[req.pages[0, 1]][:, 4:], want_k[req.pages[0, 1]][:, 4:]) and torch.equal(cache.v, want_v)


# ------------------------------------------------------------------------------------------------ adapters
ADAPTERS = [
    # rows, n, m, r, adapters, x, y0
    ("one_row", 1, 256, 128, 8, 1, "bf16", "apart"),
    ("one_row_f32", 1, 4096, 300, 16, 3, "f32", "apart"),
    ("decode", 37, 512, 640, 16, 5, "bf16", "apart"),
    ("decode_in_place", 64, 1024, 257, 32, 9, "f32", "same"),
    ("all_alike", 64, 256, 256, 16, 1, "bf16", "apart"),
    ("rows_65", 65, 256, 256, 64, 4, "bf16", "none"),
    ("odd_everything", 70, 333, 201, 13, 3, "f32", "apart"),
    ("odd_everything_bf16", 31, 77, 65, 5, 40, "bf16", "apart"),
    ("rank_1", 20, 128, 96, 1, 2, "f32", "same"),
    ("rank_128", 150, 640, 320, 128, 3, "bf16", "apart"),
    ("rank_72", 150, 640, 320, 72, 3, "f32", "apart"),
    ("prompts", 1000, 512, 384, 64, 4, "f32", "apart"),
    ("many_adapters", 3000, 96, 128, 8, 4000, "bf16", "apart"),
    ("more_adapters_than_rows", 66, 160, 64, 4, 4096, "f32", "none"),
    ("wide", 300, 2048, 3001, 40, 2, "bf16", "same"),
]


@pytest.mark.parametrize("name,rows,n,m,r,na,x,y0", ADAPTERS, ids=[c[0] for c in ADAPTERS])
@pytest.mark.parametrize("pad", [0, 3], ids=["dense", "padded"])
def test_adapters(name, rows, n, m, r, na, x, y0, pad):
    say("adapters case %s pad=%d" % (name, pad))
    g = torch.Generator(device=DEV)
    g.manual_seed(rows + n)
    X = torch.randn(rows, n + pad, generator=g, device=DEV)
    X[:, ::50] *= 30
    X = X.to(torch.bfloat16)[:, :n] if x == "bf16" else X[:, :n]
    A = (torch.randn(na, r, n, generator=g, device=DEV) / n ** 0.5).to(torch.bfloat16)
    B = torch.randn(na, m, r, generator=g, device=DEV).to(torch.bfloat16)
    scale = None if name == "decode" else torch.rand(na, generator=g, device=DEV) - 0.3
    ids = torch.randint(-1, na, (rows,), generator=g, device=DEV, dtype=torch.int32)
    if name == "all_alike":
        ids.zero_()
    elif rows > 10:
        ids[3], ids[5], ids[7] = na, 2 ** 31 - 1, -2 ** 31
    base = torch.randn(rows, m + pad, generator=g, device=DEV)
    out = base.clone() if y0 == "same" else torch.full((rows, m + pad), float("nan"), device=DEV)
    Y0 = {"same": out[:, :m], "apart": base[:, :m], "none": None}[y0]
    ctx = new_ctx()
    ctx.ensure_workspace(aser.aser_adapter_workspace_bytes(rows, n, m, r))
    ctx.check(aser.aser_adapter_forward(ctx, X, ids, A, B, scale, Y0, out[:, :m]))
    torch.cuda.synchronize()
    y = np.zeros((rows, m)) if y0 == "none" else f64(base[:, :m])
    want, size = orc.adapters(f64(X), ids.cpu().numpy(), f64(A), f64(B), None if scale is None else f64(scale), y)
    got = f64(out[:, :m])
    bar = 2.0 ** -23 * (n / 32 + r / 32 + 64) * size
    say("%s: largest error / bound %.3f, relative %.2e" % (name, (np.abs(got - want) / np.maximum(bar, 1e-30)).max(), np.linalg.norm(got - want) / np.linalg.norm(want)))
    assert (np.abs(got - want) <= bar).all()
    assert np.linalg.norm(got - want) <= 1e-6 * np.linalg.norm(want)
    bare = (ids < 0) | (ids >= na)
    if y0 != "none":
        assert torch.equal(out[bare, :m], base[bare, :m])
    if pad:
        assert torch.equal(out[:, m:], base[:, m:]) if y0 == "same" else out[:, m:].isnan().all()


def test_adapters_repeat():
    """The same bits from call to call and for a row whatever its neighbours are."""
    say("adapters repeat")
    g = torch.Generator(device=DEV)
    g.manual_seed(5)
    X = torch.randn(200, 512, generator=g, device=DEV)
    A = (torch.randn(6, 16, 512, generator=g, device=DEV) / 20).to(torch.bfloat16)
    B = torch.randn(6, 256, 16, generator=g, device=DEV).to(torch.bfloat16)
    ids = torch.randint(-1, 6, (200,), generator=g, device=DEV, dtype=torch.int32)
    ctx = new_ctx()
    ctx.ensure_workspace(aser.aser_adapter_workspace_bytes(200, 512, 256, 16))
    results = []
    for perm in (torch.arange(200, device=DEV), torch.arange(200, device=DEV), torch.randperm(200, generator=g, device=DEV)):
        out = torch.empty(200, 256, device=DEV)
        ctx.check(aser.aser_adapter_forward(ctx, X[perm].contiguous(), ids[perm].contiguous(), A, B, None, None, out))
        torch.cuda.synchronize()
        back = torch.empty_like(out)
        back[perm] = out
        results.append(back)
    assert torch.equal(results[0], results[1]) and torch.equal(results[0], results[2])
