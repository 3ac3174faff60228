"""cts_kv_write and cts_kv_read against the oracle, bit for bit: the cache's
four arrays after a write, and the values read back."""
import numpy as np
import pytest
import torch

import paper_2407_00066_amd as cts
from oracle import block as ob

from _block_helpers import TORCH, f64, to_device, to_host, values
from _gpu_helpers import say

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,heads,d,page,pages", [(1, 1, 64, 16, 1), (1, 8, 128, 16, 4), (33, 8, 128, 16, 5),
                                                  (7, 3, 256, 32, 2), (100, 2, 64, 64, 3), (61, 5, 128, 1024, 1)])
def test_write_and_read(dtype, T, heads, d, page, pages):
    say("kv_write %s T=%d heads=%d d=%d page=%d" % (dtype, T, heads, d, page))
    rng = np.random.default_rng(T * d + heads)
    n_slots = pages * page
    slots = rng.permutation(n_slots)[:T].astype(np.int64)
    T = len(slots)
    # keys and values as slices of packed rows, with a query part before and a gap behind
    width = (2 + 2 * heads) * d + 64
    rows64, rows = values(rng, (T, width), dtype, 2.0)
    k64, v64 = (rows64[:, a * d:(a + heads) * d].reshape(T, heads, d) for a in (2, 2 + heads))
    k, v = (rows[:, a * d:(a + heads) * d].unflatten(1, (heads, d)) for a in (2, 2 + heads))
    host = ob.empty_cache(pages, page, heads, d, fill=37)            # what is not written stays
    cache = to_device(host)
    ds = torch.from_numpy(slots).cuda()
    cts.kv_write(cache, k, v, ds)
    ob.write(host, k64, v64, slots)
    for got, want, name in zip(to_host(cache), host, ("k_codes", "k_scales", "v_codes", "v_scales")):
        assert np.array_equal(got, want), name
    ask = np.concatenate((slots, [-1, n_slots, 2 ** 40, -2 ** 40, slots[0]]))
    rk, rv = ob.read(host, ask)
    for out in ("bf16", "f32"):
        gk, gv = cts.kv_read(cache, torch.from_numpy(ask).cuda(), dtype=TORCH[out])
        assert np.array_equal(f64(gk), rk) and np.array_equal(f64(gv), rv)


def test_slots_outside_are_skipped():
    rng = np.random.default_rng(5)
    slots = np.array([-1, 31, 32, 2 ** 33, 0, -2 ** 62], dtype=np.int64)
    k64, k = values(rng, (6, 2, 64), "bf16")
    v64, v = values(rng, (6, 2, 64), "bf16")
    host = ob.empty_cache(2, 16, 2, 64, fill=1)
    cache = to_device(host)
    say("kv_write slots outside")
    cts.kv_write(cache, k, v, torch.from_numpy(slots).cuda())
    ob.write(host, k64, v64, slots)
    assert all(np.array_equal(a, b) for a, b in zip(to_host(cache), host))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_extreme_blocks(dtype):
    """Ties, zeros of both signs, the largest and smallest values of the type, blocks with NaN or an infinity."""
    big = 3.3895313892515355e38
    blocks = [np.zeros(32), -np.zeros(32), np.resize([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.0], 32),
              -np.resize([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 7.0], 32), np.full(32, big), np.full(32, -big),
              np.full(32, 2.0 ** 126), np.resize([2.0 ** -126, 2.0 ** -127, 0], 32), np.resize([2.0 ** -133, 0], 32),
              np.resize([1.0, 2.0 ** -30, -2.0 ** -100], 32), np.resize([1.0] * 31 + [np.nan], 32),
              np.resize([np.inf] + [1.0] * 31, 32), np.resize([-np.inf] * 31 + [np.nan], 32), np.resize([7.0, 6.5], 32),
              np.resize([6.96875, 1.0], 32), np.resize([0.2490234375, 0.25, 0.251953125, 6], 32)]
    x = torch.tensor(np.stack(blocks).reshape(4, 1, 128), dtype=torch.float64).float().to(TORCH[dtype])
    host = ob.empty_cache(1, 16, 1, 128)
    cache = to_device(host)
    say("kv_write extreme blocks %s" % dtype)
    cts.kv_write(cache, x.cuda(), x.flip(0).contiguous().cuda(), torch.arange(4, device="cuda"))
    ob.write(host, x.double().numpy(), x.flip(0).double().numpy(), range(4))
    assert all(np.array_equal(a, b) for a, b in zip(to_host(cache)[1::2], host[1::2]))
    want = ob.read(host, range(4))
    for got, ref in zip(cts.kv_read(cache, torch.arange(4, device="cuda"), dtype=torch.float32), want):
        assert np.array_equal(f64(got), ref, equal_nan=True)


def test_cache_past_32_bits():
    """Slots whose bytes lie past 2^31 and 2^32."""
    pages, page, heads, d = 1100, 1024, 32, 128                     # 2.3 GB of key codes
    cache = cts.kv_cache(pages, page, heads, d)
    n = pages * page
    slots = torch.tensor([0, n // 2 + 3, n - 1, n - 1023], device="cuda")
    rng = np.random.default_rng(6)
    k64, k = values(rng, (4, heads, d), "bf16")
    v64, v = values(rng, (4, heads, d), "bf16")
    say("kv_write past 32 bits")
    cts.kv_write(cache, k, v, slots)
    gk, gv = cts.kv_read(cache, slots)
    for got, x in ((gk, k64), (gv, v64)):
        assert np.array_equal(f64(got), ob.dequantize(*ob.quantize(x)))
    assert int(torch.count_nonzero(cache.k_scales)) == 4 * heads * d // 32


def test_outputs_in_rows_and_zero_tokens():
    cache = cts.kv_cache(2, 16, 2, 64)
    none = torch.empty((0, 2, 64), dtype=torch.bfloat16, device="cuda")
    empty = torch.empty(0, dtype=torch.int64, device="cuda")
    cts.kv_write(cache, none, none, empty)
    assert cts.kv_read(cache, empty)[0].shape == (0, 2, 64)
    rng = np.random.default_rng(7)
    _, k = values(rng, (5, 2, 64), "bf16")
    slots = torch.tensor([3, 9, 31, 16, 0], device="cuda")
    cts.kv_write(cache, k, k, slots)
    out = torch.full((5, 3, 2, 64), 9.0, dtype=torch.float32, device="cuda")
    cts.kv_read(cache, slots, k_out=out[:, 0], v_out=out[:, 2])
    want = cts.kv_read(cache, slots, dtype=torch.float32)
    assert torch.equal(out[:, 0], want[0]) and torch.equal(out[:, 2], want[1]) and bool((out[:, 1] == 9.0).all())
