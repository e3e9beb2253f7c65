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
