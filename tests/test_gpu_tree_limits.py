"""cts_kv_tree_attention where its bounds, or its tokens, come to more work than 31 bits count."""
import numpy as np
import pytest
import torch

import paper_2407_00066_amd as cts

from _draft_helpers import check, make
from _gpu_helpers import say
from test_gpu_tree_rows import _uneven
from test_gpu_tree_schedules import _plan, _widen

pytestmark = pytest.mark.gpu


# 2^20 tokens at most: units counted one by one, by fours, under a window, and tiles that are too many to cut
@pytest.mark.parametrize("B,kvh,heads,d,most,max_q,window,plan", [
    (64, 8, 32, 128, 16, 64, 0, (64, "cut", 4)), (250, 8, 32, 64, 3, 128, 0, (64, "cut", 4)),
    (64, 8, 32, 64, 16, 64, 4096, (64, "by work", 4)), (2100, 1, 4, 64, 6, 8, 0, (32, "whole", 4))])
def test_loose_bounds(B, kvh, heads, d, most, max_q, window, plan):
    n_q, n_past = _uneven(B, most, 90, [(0, 3000), (B // 2, 5000), (5, 700)], B + d)
    c = _widen(make(n_q, n_past, heads, kvh, d, 16, seed=B, words=max_q // 32 or 1), 65536)
    c["max_q"] = max_q
    assert _plan(c, window) == plan
    check(c, window)


def test_more_work_than_31_bits_count():
    """Two sequences of about 2^30 tokens (of few pages).  Queries of zero weigh all tokens alike; the values of a 64th of a
    sequence's tokens have one element of their own, so that an output counts them."""
    page, cols, kvh, heads, d, n = 1024, 2 ** 20, 8, 32, 64, 16
    cache = cts.kv_cache(256, page, kvh, d)
    cache.v_scales.fill_(127)
    slots = torch.arange(256 * page, device="cuda")
    v = torch.zeros(256 * page, kvh, d, dtype=torch.bfloat16, device="cuda")
    v[slots, :, slots // (4 * page)] = 6                         # page p: element p / 4
    cts.kv_write(cache, torch.zeros_like(v), v, slots)
    rng = np.random.default_rng(0)
    table = np.arange(cols) // (cols // 64) * 4 + rng.integers(0, 4, (2, cols))
    lens = [2 ** 30, 2 ** 30 - 123456789]
    i32 = lambda a: torch.from_numpy(np.ascontiguousarray(a, np.int32)).cuda()
    q = torch.zeros(2 * n, heads, d, dtype=torch.bfloat16, device="cuda")
    mask = torch.full((2 * n, 1), -1, dtype=torch.int32, device="cuda")
    assert cts.kv_tree_attention_plan(q, cache, torch.zeros(2, 1).expand(2, cols), n, 2 ** 30) == (64, "cut", 4)
    say("kv_tree_attention over 2 x 2^30 tokens")
    out = cts.kv_tree_attention(q, cache, i32(table), i32(lens), mask, q_start=i32([0, n, 2 * n]), max_q=n).double().cpu()
    for b, length in enumerate(lens):
        count = np.clip(length - np.arange(64) * 2 ** 24, 0, 2 ** 24)
        want = torch.from_numpy(6.0 * count / length)
        # half a step of the output; sums of these counts are exact but for the last ones over pieces
        assert bool(((out[b * n:(b + 1) * n] - want).abs() <= 1.01 * 2.0 ** -8 * want).all())
