"""cts_rotary beside a copy, and cts_kv_append beside the two calls that it stands for: neither may fall behind by far.
The bounds are wide (the calls take two thirds of them), the times are the least of many replays."""
import pytest
import torch

import paper_2407_00066_amd as cts

from _gpu_helpers import say

pytestmark = pytest.mark.gpu


def _least(f, calls=10, replays=25):
    """The least time of a call in a graph of `calls`, in us."""
    f()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        for _ in range(calls):
            f()
    best = float("inf")
    for _ in range(replays):
        a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        a.record()
        g.replay()
        b.record()
        b.synchronize()
        best = min(best, a.elapsed_time(b) * 1e3 / calls)
    return best


def _inputs(T, heads, kvh, d, dtype):
    rows = torch.randn(T, heads + 2 * kvh, d, device="cuda").to(dtype)
    angle = torch.rand(4096, d // 2, device="cuda")
    pos = torch.randint(0, 4096, (T,), device="cuda", dtype=torch.int32)
    return rows, angle.cos(), angle.sin(), pos


@pytest.mark.parametrize("T,heads,kvh,d", [(2000, 32, 8, 128), (4000, 16, 16, 64)])
def test_rotary_keeps_pace_with_a_copy(T, heads, kvh, d):
    """Queries and keys turned on one axis take 1.3 to 1.5 times a copy of them (entries of the launch's arrays found by
    comparing made it 3)."""
    rows, cos, sin, pos = _inputs(T, heads, kvh, d, torch.bfloat16)
    both = rows[:, :heads + kvh].contiguous()
    q_out, k_out, other = torch.empty_like(rows[:, :heads]), torch.empty_like(rows[:, :kvh]), torch.empty_like(both)
    say("rotary beside a copy, T=%d" % T)
    copy = _least(lambda: other.copy_(both))
    turned = _least(lambda: cts.rotary(rows[:, :heads], rows[:, heads:heads + kvh], cos, sin, pos, q_out=q_out, k_out=k_out))
    say("copy %.1f us, rotary %.1f" % (copy, turned))
    assert turned <= 2 * copy


@pytest.mark.parametrize("T,interleaved,dtype", [(1600, True, torch.float32), (1600, False, torch.float32), (1600, True, torch.bfloat16),
                                                 (1600, False, torch.bfloat16), (64, False, torch.bfloat16)])
def test_append_keeps_pace_with_its_parts(T, interleaved, dtype):
    """One call of kv_append takes no longer than rotary and kv_write (0.6 to 0.8 of them; in fp32, interleaved, with streaming
    stores 1.5)."""
    rows, cos, sin, pos = _inputs(T, 32, 8, 128, dtype)
    q, k, v = rows[:, :32], rows[:, 32:40], rows[:, 40:]
    q_out, k_out = torch.empty(T, 32, 128, dtype=dtype, device="cuda"), torch.empty(T, 8, 128, dtype=dtype, device="cuda")
    cache, slots = cts.kv_cache(T // 16 + 1, 16, 8, 128), torch.randperm(T, device="cuda")

    def parts():
        cts.rotary(q, k, cos, sin, pos, interleaved=interleaved, q_out=q_out, k_out=k_out)
        cts.kv_write(cache, k_out, v, slots)
    say("append beside rotary and write, T=%d %s interleaved=%d" % (T, dtype, interleaved))
    two = _least(parts)
    one = _least(lambda: cts.kv_append(cache, q, k, v, slots, cos, sin, pos, interleaved=interleaved, q_out=q_out))
    say("parts %.1f us, append %.1f" % (two, one))
    assert one <= 1.1 * two
