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
