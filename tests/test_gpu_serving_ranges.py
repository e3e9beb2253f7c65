"""The serving operators at the ends of their ranges: values, lengths and numbers of requests that ordinary batches do not reach.

Bounds are those of test_gpu_serving.py unless a test derives its own.
"""
import numpy as np
import pytest
import torch

import paper_2411_07762_amd as aser
from oracle import serving_oracle as orc

from gpu_util import DEV, new_ctx
from test_gpu_parity import say
from test_gpu_serving import BF16, Requests, attend, check_attention, f64, make_cache, numbers

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("sinks", [0, 3])
@pytest.mark.parametrize("window", [2 ** 31 - 1, 2 ** 31 - 7, 41])
@pytest.mark.parametrize("new", [[6, 1, 3], [150, 1, 70]], ids=["few", "prompt"])
def test_attention_under_a_window_beyond_every_key(new, window, sinks):
    """The widest windows, and one just above the longest request, beside tokens in front of position 0: as without a window."""
    say("attention widest window %d sinks=%d %s" % (window, sinks, new))
    req = Requests(new, [2, 40, 33], 16)
    cache = make_cache(req, 2, 64, False, 9)
    q, out = attend(req, cache, 4, window=window, sinks=sinks)
    check_attention("window %d" % window, req, cache, 4, q, out, window=window, sinks=sinks)
    assert torch.equal(out, attend(req, cache, 4)[1])


# ------------------------------------------------------------------------------------------------ attention
@pytest.mark.parametrize("int8", [False, True], ids=["bf16", "int8"])
@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("new", [1, 70], ids=["few", "prompt"])
@pytest.mark.parametrize("power", [34, 101])
@pytest.mark.parametrize("sign", [1.0, -1.0])
def test_attention_where_all_logits_are_far_from_zero(sign, power, new, d, int8):
    """All visible keys have one logit, of about 2^34 d or 2^101 d and either sign: every one counts the same.  Then one key has the largest: it alone counts."""
    say("attention far logits %+.0f 2^%d new=%d d=%d int8=%s" % (sign, power, new, d, int8))
    kv = 1500
    req = Requests([new], [kv], 32)
    cache = make_cache(req, 1, d, int8, 10)
    q = (2.0 ** (power // 2) * (1 + torch.arange(d, device=DEV) % 97 / 128)).to(torch.bfloat16).repeat(new, 4)
    high = power - power // 2
    for one in (False, True):
        if int8:
            cache.k.fill_(int(sign) * 64)
            cache.k_scale.fill_(2.0 ** (high - 6))
        else:
            cache.k.fill_(sign * 2.0 ** high)
        if one:                                            # key 77: half of the others' negative logit, twice their positive one
            f = 2.0 if sign > 0 else 0.5
            if int8:
                cache.k_scale[req.pages[0, 77 // 32], :, 77 % 32] *= f
            else:
                cache.k[req.pages[0, 77 // 32], :, 77 % 32] *= f
        out = torch.empty_like(q)
        ctx, batch = new_ctx(), req.batch()
        ctx.ensure_workspace(aser.aser_paged_attention_workspace_bytes(cache, batch, 4))
        ctx.check(aser.aser_paged_attention(ctx, q, cache, batch, out, scale=1.0))
        torch.cuda.synchronize()
        check_attention("one logit" if not one else "one key", req, cache, 4, q, out, scale=1.0)


# ------------------------------------------------------------------------------------------------ append
@pytest.mark.parametrize("norm", [False, True], ids=["plain", "norm"])
def test_append_to_an_int8_cache_keeps_what_is_not_finite(norm):
    """A head with a NaN or an infinity has the scale NaN, and attention that sees it gives NaN; every other head is stored as without it."""
    say("append int8 not finite norm=%s" % norm)
    new, d, kv_heads, heads = [7, 1], 64, 2, 4
    req = Requests(new, [20, 40], 16)
    g = torch.Generator(device=DEV)
    g.manual_seed(6)
    q, k, v = (torch.randn(8, n * d, generator=g, device=DEV) for n in (heads, kv_heads, kv_heads))
    kn = torch.ones(d, device=DEV) if norm else None
    bad_k, bad_v = torch.zeros(8, kv_heads, dtype=torch.bool), torch.zeros(8, kv_heads, dtype=torch.bool)
    results = []
    for spoil in (False, True):
        if spoil:
            k[1, :d], k[2, d + 5], k[3, 11], v[4, d + 63], v[5, 0] = float("nan"), float("nan"), float("inf"), -float("inf"), float("nan")
            bad_k[1, 0] = bad_k[2, 1] = bad_k[3, 0] = bad_v[4, 1] = bad_v[5, 0] = True
        cache = make_cache(req, kv_heads, d, True, 12)
        out = torch.empty(8, heads * d, dtype=torch.bfloat16, device=DEV)
        ctx = new_ctx()
        ctx.check(aser.aser_kv_append(ctx, q, k, v, cache, req.batch(), out, k_norm=kn))
        torch.cuda.synchronize()
        results.append((cache, out))
    (clean, _), (cache, out) = results
    at = torch.cat([torch.arange(13, 20), torch.tensor([39])])
    page = torch.from_numpy(np.concatenate([req.pages[0][np.arange(13, 20) // 16], req.pages[1][39 // 16:39 // 16 + 1]])).long()
    for name, bad in (("k", bad_k), ("v", bad_v)):
        scale, ref = (getattr(c, name + "_scale").cpu()[page, :, at % 16] for c in (cache, clean))
        codes, ref_codes = (getattr(c, name).cpu()[page, :, at % 16] for c in (cache, clean))
        assert scale[bad].isnan().all()
        assert torch.equal(scale[~bad], ref[~bad]) and torch.equal(codes[~bad], ref_codes[~bad])
    q, got = attend(req, cache, heads)
    got = f64(got).reshape(8, kv_heads, heads // kv_heads, d)
    assert np.isnan(got[:7][[1, 2, 3, 4, 5, 6]][:, 0]).all() and np.isnan(got[2:7, 1]).all()
    assert np.isfinite(got[7]).all()


# ------------------------------------------------------------------------------------------------ adapters
def adapt(X, ids, A, B, scale=None, Y0=None):
    rows, m = X.shape[0], B.shape[1]
    out = torch.full((rows, m), 7.0, device=DEV)
    ctx = new_ctx()
    ctx.ensure_workspace(aser.aser_adapter_workspace_bytes(rows, X.shape[1], m, A.shape[1]))
    ctx.check(aser.aser_adapter_forward(ctx, X, ids, A, B, scale, Y0, out))
    torch.cuda.synchronize()
    return out


@pytest.mark.parametrize("r", [13, 72])
@pytest.mark.parametrize("rows", [5, 70])
@pytest.mark.parametrize("scale", [1e-37, 1e-36, 1e-33, 1e-30, 1e30])
def test_adapters_keep_all_bits_at_any_scale(scale, rows, r):
    """Inputs, or inner products alone, of a size whose lower bits three bf16 terms do not hold: the bound of the other sizes.  (The fp32 instruction
    adds n / 4 + r / 4 times instead of n / 32 + r / 32, each time at half an ulp: 87 to 102 of the 149 halves that the bound has.)"""
    say("adapters at %g, %d rows" % (scale, rows))
    n, m, na = 333, 201, 3
    g = torch.Generator(device=DEV)
    g.manual_seed(rows)

    def rand(*shape):
        return torch.randn(*shape, generator=g, device=DEV)

    ids = torch.randint(0, na, (rows,), generator=g, device=DEV, dtype=torch.int32)
    for x_scale, a_scale in ((scale, 1.0), (1.0, scale)):
        X, A, B = rand(rows, n) * x_scale, (rand(na, r, n) * a_scale).to(torch.bfloat16), (rand(na, m, r) / scale).to(torch.bfloat16)
        got = f64(adapt(X, ids, A, B))
        want, size = orc.adapters(f64(X), ids.cpu().numpy(), f64(A), f64(B), None, np.zeros((rows, m)))
        bar = 2.0 ** -23 * (n / 32 + r / 32 + 64) * size
        rel = np.linalg.norm(got - want) / np.linalg.norm(want)
        say("x %g, A %g: largest error / bound %.3f, relative %.2e" % (x_scale, a_scale, (np.abs(got - want) / bar).max(), rel))
        assert (np.abs(got - want) <= bar).all()
        assert rel <= 1e-6


@pytest.mark.parametrize("rows", [9, 100])
@pytest.mark.parametrize("x", ["f32", "bf16"])
@pytest.mark.parametrize("n,r", [(256, 16), (259, 13)])
def test_adapters_of_inputs_that_are_not_finite(n, r, x, rows):
    """An infinity gives an infinity where the formula does, a NaN a NaN; the largest finite values, which round to an infinity in bf16, give what they
    should; and rows beside them keep their bits."""
    say("adapters not finite n=%d r=%d %s %d rows" % (n, r, x, rows))
    m, na = 130, 2
    g = torch.Generator(device=DEV)
    g.manual_seed(n)
    A, B = (torch.rand(na, *s, generator=g, device=DEV) * 1e-3 + 1e-4 for s in ((r, n), (m, r)))
    A, B = A.to(torch.bfloat16), B.to(torch.bfloat16)
    X = torch.randn(rows, n, generator=g, device=DEV)
    X = X.to(torch.bfloat16) if x == "bf16" else X
    ids = torch.arange(rows, device=DEV, dtype=torch.int32) % na
    y0 = torch.randn(rows, m, generator=g, device=DEV)
    before = adapt(X, ids, A, B, None, y0)
    inf = float("inf")
    X[0, 3], X[1, n - 1], X[2, 5], X[3, 0], X[3, 40] = inf, -inf, float("nan"), inf, -inf
    X[4, 7] = 3.4e38 if x == "f32" else torch.finfo(torch.bfloat16).max
    X[5, 9] = -torch.finfo(X.dtype).max
    got = adapt(X, ids, A, B, None, y0)
    assert torch.equal(got[6:], before[6:])
    got = f64(got)
    assert (got[0] == inf).all() and (got[1] == -inf).all() and np.isnan(got[2:4]).all()
    want, size = orc.adapters(f64(X[4:6]), ids[4:6].cpu().numpy(), f64(A), f64(B), None, f64(y0[4:6]))
    assert (np.abs(got[4:6] - want) <= 2.0 ** -23 * (n / 32 + r / 32 + 64) * size).all()


@pytest.mark.parametrize("kv_heads,d", [(1, 64), (2, 64), (1, 128), (2, 256)])
def test_attention_of_more_requests_than_a_wavefront_looks_at_once(kv_heads, d):
    """130 requests, most of them single tokens, prompts on both sides of numbers 64 and 128; one key/value head: keys of prompts in parts."""
    say("attention of 130 requests, %d key/value heads of %d" % (kv_heads, d))
    new, kv = [1] * 130, [1 + (37 * s) % 190 for s in range(130)]
    for s, n in ((3, 40), (62, 33), (63, 70), (64, 40), (65, 2), (100, 0), (127, 35), (128, 130), (129, 41)):
        new[s], kv[s] = n, n + 900 + s
    req = Requests(new, kv, 32, seed=kv_heads)
    cache = make_cache(req, kv_heads, d, False, 21)
    q, out = attend(req, cache, 4 * kv_heads)
    check_attention("130 requests", req, cache, 4 * kv_heads, q, out)
    q, out = attend(req, cache, 4 * kv_heads, window=50, sinks=3)
    check_attention("130 requests, window", req, cache, 4 * kv_heads, q, out, window=50, sinks=3)


@pytest.mark.parametrize("kv,heads,kv_heads,d,int8", [(70001, 4, 1, 64, False), (70001, 2, 1, 64, True), (33003, 8, 2, 128, False), (40000, 2, 1, 256, False)])
def test_attention_in_more_parts_than_a_wavefront_joins_at_once(kv, heads, kv_heads, d, int8):
    """One token over an axis that is cut into 115 to 244 parts."""
    say("attention over %d keys" % kv)
    req = Requests([1], [kv], 64)
    cache = make_cache(req, kv_heads, d, int8, 4)
    q, out = attend(req, cache, heads)
    check_attention("%d keys" % kv, req, cache, heads, q, out)


@pytest.mark.filterwarnings("ignore:invalid value encountered:RuntimeWarning")    # codes times scales that nobody sees
@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("new", [[1, 2], [100, 37]], ids=["few", "prompt"])
def test_attention_ignores_int8_scales_that_nobody_sees(new, d):
    """NaN and infinities as scales of slots past the request's tokens, of keys that left the window and of pages that the table does not name."""
    say("attention unseen scales %s d=%d" % (new, d))
    req = Requests(new, [200, 45], 16, spare=3)
    for window, sinks in ((48, 4), (0, 0)):
        cache = make_cache(req, 2, d, True, 7)
        used = np.zeros((req.n_pages, req.page), bool)
        for s in range(2):
            low = req.kv[s] - new[s] - window + 1 if window else 0
            for p in range(req.kv[s]):
                used[req.pages[s, p // 16], p % 16] = p >= low or p < sinks
        hide = torch.from_numpy(~used).to(DEV)[:, None, :]
        cache.k_scale.masked_fill_(hide, float("nan"))
        cache.v_scale.masked_fill_(hide, float("inf"))
        cache.v_scale[:, 1].masked_fill_(hide[:, 0], float("nan"))
        q, out = attend(req, cache, 8, window=window, sinks=sinks)
        check_attention("unseen scales", req, cache, 8, q, out, window=window, sinks=sinks)
    for at, bad in ((3, -1), (5, req.n_pages), (7, 2 ** 31 - 1)):
        req.pages[0, at] = bad
    cache = make_cache(req, 2, d, True, 8)
    cache.k_scale[0] = float("nan")                        # the page that is read in place of one that is not there
    cache.v_scale[0] = float("inf")
    free = sorted(set(range(1, req.n_pages)) - set(req.pages.reshape(-1).tolist()))
    req.pages[req.pages == 0] = free[0]
    q, out = attend(req, cache, 8)
    check_attention("missing pages", req, cache, 8, q, out)


TWO_TERMS = [
    # new, kv, heads, kv_heads, d, page, int8, window, sinks
    ([1], [77], 32, 8, 128, 64, False, 0, 0),
    ([1, 1], [5003, 60], 16, 4, 128, 32, False, 0, 0),
    ([1] * 3, [2049, 31, 400], 8, 2, 256, 64, False, 0, 0),
    ([4, 1, 7, 2], [60, 9, 30, 900], 8, 4, 64, 32, False, 0, 0),
    ([1, 1, 2], [4097, 1300, 50], 32, 4, 64, 16, True, 0, 0),
    ([1] * 5, [31, 32, 33, 64, 700], 16, 4, 128, 128, True, 0, 0),
    ([1, 3, 1], [40, 500, 4001], 8, 2, 128, 32, False, 64, 4),
]


@pytest.mark.parametrize("new,kv,heads,kv_heads,d,page,int8,window,sinks", TWO_TERMS, ids=[str(i) for i in range(len(TWO_TERMS))])
@pytest.mark.parametrize("beside", [False, True], ids=["alone", "beside_a_prompt"])
def test_few_rows_keep_probabilities_to_two_terms(new, kv, heads, kv_heads, d, page, int8, window, sinks, beside):
    """Requests of at most 64 rows: the result's rounding (2^-8 of it), what two bf16 terms leave of the probabilities (2^-16 of sum p |v|) and fp32 arithmetic
    (1e-4 of that sum).  Over all outputs the roundings of the results come to 1.5e-3 to 1.7e-3 of the norm: their mean square is a third of the largest
    one's over the binades' mean.  The same sums with probabilities rounded once to bf16 do not pass."""
    say("attention two terms %s %s beside=%s" % (new, kv, beside))
    if beside:
        new, kv = list(new) + [100], list(kv) + [120]
    req = Requests(new, kv, page)
    cache = make_cache(req, kv_heads, d, int8, 5)
    q, out = attend(req, cache, heads, window=window, sinks=sinks)
    k, v = numbers(cache)
    rows = slice(0, int(req.start[len(new) - beside]))
    qn = f64(q).reshape(req.tokens, heads, d)
    want, size = orc.attention(qn, k, v, req.pages, req.start, req.kv_len, d ** -0.5, window, sinks)

    def passes(got):
        err = np.abs(got - want)[rows]
        rel = np.linalg.norm(err) / np.linalg.norm(want[rows])
        bar = BF16 * np.abs(want[rows]) + (2.0 ** -16 + 1e-4) * size[rows]
        say("largest error / bound %.2f, relative %.2e" % ((err / bar).max(), rel))
        return bool((err <= bar).all()) and rel <= 1.9e-3

    assert passes(f64(out).reshape(want.shape))

    def rounded(x):
        return torch.from_numpy(np.asarray(x, np.float32)).to(torch.bfloat16).float().numpy().astype(np.float64)

    once = np.zeros_like(want)
    for s in range(len(new) - beside):
        n = kv[s]
        j = np.arange(n)
        at = req.pages[s][j // page]
        ok = orc.visible(orc.positions_of(req.start, req.kv_len, s), n, window, sinks)
        for h in range(heads):
            kh, vh = k[at, h * kv_heads // heads, j % page], v[at, h * kv_heads // heads, j % page]
            logits = np.where(ok, qn[req.start[s]:req.start[s + 1], h] @ kh.T * d ** -0.5, -np.inf)
            p = np.exp(logits - logits.max(1, keepdims=True))
            once[req.start[s]:req.start[s + 1], h] = rounded(rounded(p) @ vh / p.sum(1, keepdims=True))
    assert not passes(once)
