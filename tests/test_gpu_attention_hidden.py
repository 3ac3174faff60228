"""What a query does not see leaves no trace in its row, whatever bytes the cache
holds there: scale bytes past the written ones (253 and 254 put some magnitudes
past the largest float) behind the causal mask, before a window and past the end."""
import numpy as np
import pytest
import torch

from oracle import block as ob

from _block_helpers import ROUND, assert_within
from _gpu_helpers import say
from test_gpu_kv_attention import WEIGHTS, call, make

pytestmark = pytest.mark.gpu


def _spoil(c, b, t, byte, code):
    """Token t of sequence b: every scale this byte, every element this code."""
    kc, ks, vc, vs = c["cache"]
    page = kc.shape[2]
    p, o = int(c["table"][b][t // page]), t % page
    ks[p, :, o] = byte
    kc[p, :, o] = code * 17
    vs[p, :, o // 4, :, o % 4] = byte
    vc[p, :, o // 4, :, o % 4] = code * 17


@pytest.mark.parametrize("byte,code", [(253, 7), (254, 4), (254, 15), (255, 7), (252, 7)])
@pytest.mark.parametrize("dtype,d,n_q,window", [
    ("bf16", 64, 1, 0), ("bf16", 128, 1, 9), ("f32", 256, 1, 0), ("bf16", 128, 14, 0), ("f32", 64, 9, 6), ("bf16", 256, 9, 0),
    ("bf16", 64, 70, 0), ("bf16", 128, 130, 30), ("bf16", 256, 50, 0), ("f32", 128, 50, 20)])
def test_bytes_past_the_written_ones(dtype, d, n_q, window, byte, code):
    page, L = 32, n_q + 39
    c = make([n_q], [L], 4, 2, d, page, dtype, seed=d + n_q)
    want, mag, soft = ob.attention(c["q64"], c["cache"], c["table"], c["n_kv"], c["q_start"], d ** -0.5, window)
    spoiled = list(range(L, -(-L // page) * page))                      # past the end, in the last page
    if n_q > 4:
        spoiled += [L - 2, L - 2 - n_q // 3]                            # seen by later queries only
    if window:
        spoiled += [0, 3]                                               # before the window of most
    for t in spoiled:
        _spoil(c, 0, t, byte, code)
    say("kv_attention %s d=%d n=%d window=%d byte %d code %d" % (dtype, d, n_q, window, byte, code))
    out = call(c, window)
    pos = L - n_q + np.arange(n_q)
    first = np.maximum(0, pos - window + 1) if window else 0 * pos
    clean = np.array([not any(f <= t <= p for t in spoiled) for f, p in zip(first, pos)])
    assert clean.sum() >= min(n_q, 3)
    w, m, s = want[clean], mag[clean], soft[clean]
    got = out[torch.from_numpy(clean).cuda()]
    assert_within(got, w, 1.01 * (ROUND[dtype] * np.abs(w) + WEIGHTS[dtype] * m + s) + 1e-30, "rows that see none of it")
