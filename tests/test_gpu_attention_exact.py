"""cts_kv_attention where the result is known far better than a product's
roundings allow in general: values that are all the same, and zero queries, whose
weights are all one."""
import numpy as np
import pytest
import torch

from _gpu_helpers import say
from test_gpu_kv_attention import call, make

pytestmark = pytest.mark.gpu


# prompts, few rows (16-row tiles), long contexts in pieces, prompts in pieces
SHAPES = [([40], [40], 0, None), ([1, 5, 64], [90, 77, 64], 0, None), ([65, 300, 17], [65, 300, 500], 0, None),
          ([200], [333], 50, None), ([1, 2], [3000, 10], 0, 4000), ([70, 128], [2500, 3000], 0, None)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("n_q,n_kv,window,max_kv", SHAPES)
def test_equal_values(n_q, n_kv, window, max_kv, d, dtype):
    """All tokens hold the same value: so does the output, whatever the weights and
    however they are rounded, for a row's length is the sum of its weights as they
    are multiplied.  The sums of up to 3000 weights and their quotient carry at most
    3100 x 2^-24 of it, less than half a step of bf16: bf16 outputs are exact."""
    if dtype == "f32" and max(n_q) > 200:
        n_q, n_kv = [min(n, 100) for n in n_q], n_kv
    c = make(n_q, n_kv, 8, 2, d, 16, dtype, seed=d + len(n_q))
    codes = np.random.default_rng(d).integers(0, 16, (2, d), dtype=np.uint8)      # a head's value
    mag = np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6])[codes & 7] * np.where(codes >= 8, -1, 1)
    by = (codes[:, 0::2] | (codes[:, 1::2] << 4)).reshape(2, d // 8, 1, 4)
    c["cache"][2][...] = by[None, :, None]
    c["cache"][3][...] = 127
    say("kv_attention equal values %s d=%d q=%s kv=%s" % (dtype, d, n_q, n_kv))
    out = call(c, window, **({} if max_kv is None else {"max_kv": max_kv}))
    want = torch.from_numpy(np.repeat(mag, 4, axis=0)).cuda().expand(out.shape)
    if dtype == "bf16":
        assert torch.equal(out.double(), want)
    else:
        assert bool(((out.double() - want).abs() <= 3100 * 2.0 ** -24 * want.abs()).all())
