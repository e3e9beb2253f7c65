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
