"""The drafted-token calls' binding on the GPU: what it does with arguments left out, and what it returns."""
import numpy as np
import pytest
import torch

import paper_2407_00066_amd as cts

from _block_helpers import assert_within, to_device
from _draft_helpers import bound, expected, i32, make
from _gpu_helpers import say

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n_q,words", [([40], 1), ([40, 3], 1), ([20, 13], 1), ([3, 65], 2), ([300, 300], 18)])
def test_a_mask_of_too_few_words_without_max_q(n_q, words):
    """Without max_q all rows may be one sequence's: a mask without a bit for each, or more rows than a sequence may have, is
    refused, since rows past its bits would be left unwritten."""
    c = make(n_q, [30] * len(n_q), 4, 2, 64, 16, seed=sum(n_q), words=max(words, -(-max(n_q) // 32)))
    cache, table, n_kv, start = to_device(c["cache"]), i32(c["table"]), i32(c["n_kv"]), i32(c["q_start"])
    mask = i32(c["mask"][:, :words])
    say("kv_tree_attention without max_q, q=%s words=%d" % (n_q, words))
    with pytest.raises(ValueError, match="max_q"):
        cts.kv_tree_attention(c["q"], cache, table, n_kv, mask, q_start=start)
    if max(n_q) <= 32 * words:                                   # with max_q it is taken
        out = cts.kv_tree_attention(c["q"], cache, table, n_kv, mask, q_start=start, max_q=max(n_q))
        want, mag, soft = expected(c)
        assert_within(out, want, bound(c, want, mag, soft), "with max_q")


@pytest.mark.parametrize("n_q", [[3, 1, 6], [32], [16, 0, 16], [1, 1]])
def test_all_drafts_without_max_q(n_q):
    c = make(n_q, [70, 5, 0][:len(n_q)], 4, 2, 64, 16, seed=sum(n_q))
    # what torch hands out next held NaN: a row that is left out cannot pass for a result
    spare = [torch.full_like(c["q"], float("nan")) for _ in range(4)]
    torch.cuda.synchronize()
    del spare
    say("kv_tree_attention without max_q, q=%s" % n_q)
    out = cts.kv_tree_attention(c["q"], to_device(c["cache"]), i32(c["table"]), i32(c["n_kv"]), i32(c["mask"]), q_start=i32(c["q_start"]))
    want, mag, soft = expected(c)
    assert_within(out, want, bound(c, want, mag, soft), "without max_q")


@pytest.mark.parametrize("heads", [0, 5])
def test_append_in_place_returns_the_queries(heads):
    """kv_append gives back the queries that it was told to write, or None without queries."""
    rows = torch.randn(4, heads + 4, 64, device="cuda").bfloat16()
    q, k, v = rows[:, :heads], rows[:, heads:heads + 2], rows[:, heads + 2:]
    angle = torch.rand(9, 32, device="cuda")
    cache, at, pos = cts.kv_cache(1, 16, 2, 64), torch.arange(4, device="cuda"), i32(np.arange(4, dtype=np.int32))
    want = cts.rotary(q, None, angle.cos(), angle.sin(), pos)[0] if heads else None
    say("kv_append in place, %d heads" % heads)
    got = cts.kv_append(cache, q if heads else None, k, v, at, angle.cos(), angle.sin(), pos, q_out=q if heads else None, k_out=k)
    if heads:
        assert got.data_ptr() == q.data_ptr() and got.stride() == q.stride() and got.shape == q.shape
        assert torch.equal(got, want)
    else:
        assert got is None
