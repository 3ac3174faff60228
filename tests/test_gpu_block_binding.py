"""The decoder block's binding on the GPU: what a call does with arguments left
out, and the errors it raises."""
import numpy as np
import pytest
import torch

import paper_2407_00066_amd as cts

from _block_helpers import to_device
from _gpu_helpers import say
from test_gpu_kv_attention import call, make

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n_q,n_kv", [([3, 1, 6], [77, 1, 130]), ([70, 0, 9], [200, 5, 9]), ([1, 1], [40, 7])])
def test_attention_of_all_queries_without_max_q(n_q, n_kv):
    """q_start says how many queries there are: left out, max_q hides none of them."""
    c = make(n_q, n_kv, 4, 2, 64, 16, seed=sum(n_q))
    cache, table, n = to_device(c["cache"]), torch.from_numpy(c["table"]).cuda(), torch.from_numpy(c["n_kv"]).cuda()
    # what torch hands out next held NaN: a row that is left out cannot pass for a result
    spare = [torch.full_like(c["q"], float("nan")) for _ in range(4)]
    torch.cuda.synchronize()
    del spare
    say("kv_attention without max_q, q=%s" % n_q)
    out = cts.kv_attention(c["q"], cache, table, n, q_start=torch.from_numpy(c["q_start"]).cuda())
    want = call(c).double()
    assert not bool(torch.isnan(out).any())
    assert bool(((out.double() - want).abs() <= 2.0 ** -5 * (1 + want.abs())).all())
    assert np.array_equal(c["q_start"], np.concatenate(([0], np.cumsum(n_q))))


def test_more_rows_than_max_q_can_be():
    """Without max_q, rows past the 2^24 that one sequence can have are refused, not left out; with it they are taken."""
    T, B = 2 ** 24 + 2, 2
    q = torch.zeros(T, 1, 64, dtype=torch.bfloat16, device="cuda")
    cache = cts.kv_cache(2, 16, 1, 64)
    table = torch.tensor([[0], [1]], dtype=torch.int32, device="cuda")
    n = torch.tensor([3, 2], dtype=torch.int32, device="cuda")
    start = torch.tensor([0, 1, 3], dtype=torch.int32, device="cuda")
    say("kv_attention of %d rows" % T)
    with pytest.raises(cts.CtsError):
        cts.kv_attention(q, cache, table, n, q_start=start)
    out = torch.full_like(q, 5.0)
    cts.kv_attention(q, cache, table, n, q_start=start, max_q=B, out=out)
    assert not out[:3].any() and bool((out[3:] == 5).all())


def test_out_of_memory_keeps_its_type():
    """A program that catches torch.OutOfMemoryError around the layer's calls catches it here."""
    cache = cts.kv_cache(1, 16, 64, 256)
    slots = torch.zeros(200000, dtype=torch.int64, device="cuda")        # 2 x 13 GB in fp32
    say("kv_read past the allowed memory")
    torch.cuda.empty_cache()
    total = torch.cuda.get_device_properties(0).total_memory
    torch.cuda.set_per_process_memory_fraction((torch.cuda.memory_reserved() + (1 << 30)) / total)
    try:
        with pytest.raises(torch.OutOfMemoryError):
            cts.kv_read(cache, slots, dtype=torch.float32)
    finally:
        torch.cuda.set_per_process_memory_fraction(1.0)
    assert cts.kv_read(cache, slots[:5])[0].shape == (5, 64, 256)
