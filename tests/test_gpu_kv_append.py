"""cts_kv_append: equal by bits to cts_rotary and cts_kv_write, whose formulas the oracle has."""
import numpy as np
import pytest
import torch

import paper_2407_00066_amd as cts
from oracle import block as ob

from _block_helpers import ROUND, TORCH, assert_within, f64, to_device, to_host
from _draft_helpers import filled
from _gpu_helpers import say

pytestmark = pytest.mark.gpu


def _angles(n_pos, rot):
    a = torch.arange(n_pos, dtype=torch.float64)[:, None] * 100.0 ** (-torch.arange(rot // 2, dtype=torch.float64) / (rot // 2))
    return a.cos().float().cuda(), a.sin().float().cuda()


def _inputs(T, heads, kvh, d, rot, axes, page, dtype, seed=0):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    rows = torch.randn(T, heads + 2 * kvh, d, generator=g, device="cuda").to(TORCH[dtype])
    pages = -(-T // page) + 2
    slots = torch.randperm(pages * page, generator=g, device="cuda")[:T]
    pos = torch.randint(-2, 40, (axes, T), generator=g, device="cuda", dtype=torch.int32)
    sections = [rot // 2 - (axes - 1) * (rot // 2 // axes)] + [rot // 2 // axes] * (axes - 1)
    cache = to_device(filled(np.random.default_rng(seed), pages, page, kvh, d))
    return rows, slots, pos, sections, cache, _angles(38, rot)


def _copy(cache):
    return cts.KVCache(*(t.clone() for t in (cache.k_codes, cache.k_scales, cache.v_codes, cache.v_scales)))


def _same(a, b):
    return all(np.array_equal(x, y) for x, y in zip(to_host(a), to_host(b)))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("T,heads,kvh,d,rot,axes,page", [
    (1, 4, 1, 64, 64, 1, 16), (3, 8, 2, 128, 128, 1, 16), (33, 5, 5, 64, 32, 3, 32), (70, 4, 2, 256, 256, 2, 16),
    (7, 6, 3, 128, 16, 1, 64), (19, 2, 1, 128, 48, 2, 16), (5, 0, 4, 128, 112, 4, 16), (1200, 12, 3, 64, 64, 1, 128),
    (2500, 16, 4, 128, 128, 1, 16)])
def test_equals_rotary_and_write(T, heads, kvh, d, rot, axes, page, interleaved, dtype):
    rows, slots, pos, sections, cache, (cos, sin) = _inputs(T, heads, kvh, d, rot, axes, page, dtype, T + d)
    q, k, v = rows[:, :heads], rows[:, heads:heads + kvh], rows[:, heads + kvh:]
    if T > 2:
        slots[T // 2], slots[1] = -1, 2 ** 40                   # padding
    other, whole = _copy(cache), _copy(cache)
    say("kv_append T=%d heads=%d/%d d=%d rot=%d axes=%d %s" % (T, heads, kvh, d, rot, axes, dtype))
    want_q, want_k = cts.rotary(q if heads else None, k, cos, sin, pos, sections=sections, interleaved=interleaved)
    cts.kv_write(other, want_k, v, slots)
    got = cts.kv_append(cache, q if heads else None, k, v, slots, cos, sin, pos, sections=sections, interleaved=interleaved)
    assert (got is None and not heads) or torch.equal(got, want_q)
    assert _same(cache, other)
    # in place, the turned keys returned too; nothing else of the rows is touched
    before = rows.clone()
    assert cts.kv_append(whole, q if heads else None, k, v, slots, cos, sin, pos, sections=sections, interleaved=interleaved,
                         q_out=q if heads else None, k_out=k) is (q if heads else None) or heads
    assert torch.equal(k, want_k) and torch.equal(v, before[:, heads + kvh:]) and _same(whole, other)
    assert not heads or torch.equal(q, want_q)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_against_the_oracle(dtype):
    rows, slots, pos, sections, cache, (cos, sin) = _inputs(9, 4, 2, 128, 64, 2, 16, dtype, 3)
    host = tuple(a.copy() for a in to_host(cache))
    k_out = torch.empty(9, 2, 128, dtype=rows.dtype, device="cuda")
    say("kv_append against the oracle %s" % dtype)
    q = cts.kv_append(cache, rows[:, :4], rows[:, 4:6], rows[:, 6:], slots, cos, sin, pos, sections=sections, k_out=k_out)
    for got, x in ((q, rows[:, :4]), (k_out, rows[:, 4:6])):
        want, mag = ob.rotary(f64(x), f64(cos), f64(sin), pos.cpu().numpy(), sections)
        assert_within(got, want, 1.01 * ROUND[dtype] * np.abs(want) + 2.0 ** -22 * mag, "turned")
    ob.write(host, f64(k_out), f64(rows[:, 6:]), slots.cpu().numpy())       # (from the turned keys: a rounding may move a code)
    assert all(np.array_equal(a, b) for a, b in zip(to_host(cache), host))


@pytest.mark.parametrize("interleaved", [False, True])
def test_values_that_are_no_numbers(interleaved):
    """A NaN or an infinity makes its blocks, and those it is turned with, NaN, as the two calls do."""
    rows, slots, pos, sections, cache, (cos, sin) = _inputs(6, 2, 2, 128, 128, 1, 16, "bf16", 4)
    rows[1, 2, 5], rows[2, 3, 70], rows[3, 5, 127], rows[4] = float("nan"), float("inf"), float("-inf"), 0
    rows[5] = 3e38
    other = _copy(cache)
    k, v = rows[:, 2:4], rows[:, 4:]
    say("kv_append of NaN")
    q, k2 = cts.rotary(rows[:, :2], k, cos, sin, pos, interleaved=interleaved)
    cts.kv_write(other, k2, v, slots)
    got = cts.kv_append(cache, rows[:, :2], k, v, slots, cos, sin, pos, interleaved=interleaved)
    assert _same(cache, other) and torch.equal(got.view(torch.int16), q.view(torch.int16))


def test_slots_past_32_bits():
    """Pages whose bytes lie past 2^32."""
    n, page, kvh, d = 40000, 1024, 2, 256                       # 10.5 GB of codes of each kind
    cache = cts.kv_cache(n, page, kvh, d)
    rows, _, pos, _, _, (cos, sin) = _inputs(4, 2, kvh, d, d, 1, 16, "bf16", 5)
    slots = torch.tensor([n * page - 1, 0, 17000 * page + 5, n * page], device="cuda")
    say("kv_append past 32 bits")
    k_out = torch.empty(4, kvh, d, dtype=torch.bfloat16, device="cuda")
    cts.kv_append(cache, rows[:, :2], rows[:, 2:4], rows[:, 4:], slots, cos, sin, pos, k_out=k_out)
    small = cts.kv_cache(1, 16, kvh, d)
    at = torch.arange(4, device="cuda")
    cts.kv_write(small, k_out, rows[:, 4:], at)
    for a, b in zip(cts.kv_read(cache, slots[:3]), cts.kv_read(small, at[:3])):
        assert torch.equal(a, b)


def test_captured_with_new_values():
    """A captured call replays on what its buffers hold then."""
    rows, slots, pos, sections, cache, (cos, sin) = _inputs(20, 4, 2, 64, 64, 1, 16, "bf16", 6)
    q_out = torch.empty(20, 4, 64, dtype=torch.bfloat16, device="cuda")
    run = lambda c, out: cts.kv_append(c, rows[:, :4], rows[:, 4:6], rows[:, 6:], slots, cos, sin, pos, q_out=out)
    run(cache, q_out)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        run(cache, q_out)
    for i in range(3):
        rows.copy_(torch.randn_like(rows.float()).bfloat16())
        pos.add_(1)
        other, want = _copy(cache), torch.empty_like(q_out)
        say("kv_append replay %d" % i)
        g.replay()
        torch.cuda.synchronize()
        run(other, want)
        torch.cuda.synchronize()
        assert _same(cache, other) and torch.equal(q_out, want)


def test_refusals():
    rows, slots, pos, sections, cache, (cos, sin) = _inputs(5, 2, 2, 64, 64, 1, 16, "bf16", 7)
    q, k, v = rows[:, :2], rows[:, 2:4], rows[:, 4:]
    before = [a.copy() for a in to_host(cache)]
    for args, kw, error in [((None, k, v, slots, cos, sin, pos), dict(q_out=q), ValueError),
                            ((q, k[:, :1], v, slots, cos, sin, pos), {}, ValueError),
                            ((q.float(), k, v, slots, cos, sin, pos), {}, TypeError),
                            ((q, k, v, slots.int(), cos, sin, pos), {}, TypeError),
                            ((q, k, v, slots[:4], cos, sin, pos), {}, ValueError),
                            ((q, k, v, slots, cos.double(), sin, pos), {}, TypeError),
                            ((q, k, v, slots, cos, sin, pos), dict(sections=[16, 16]), ValueError),
                            ((q, k, v, slots, cos, sin, pos), dict(k_out=q), cts.CtsError),
                            ((q, k, v, slots, cos, sin, pos), dict(q_out=k), cts.CtsError),
                            ((q, k, v, slots, cos[:, :20].contiguous(), sin[:, :20].contiguous(), pos), {}, cts.CtsError)]:
        with pytest.raises(error):
            cts.kv_append(cache, *args, **kw)
    assert all(np.array_equal(a, b) for a, b in zip(to_host(cache), before))


@pytest.mark.parametrize("heads,kvh,dtype", [(7, 3, "bf16"), (0, 5, "bf16"), (9, 1, "f32")])
def test_odd_heads_of_many_tokens_in_place(heads, kvh, dtype):
    """Threads that take two heads where one is left over: rows are turned in place, on a stream of their own."""
    T = 6001
    rows, slots, pos, sections, cache, (cos, sin) = _inputs(T, heads, kvh, 128, 128, 1, 16, dtype, T + heads)
    q, k, v = rows[:, :heads] if heads else None, rows[:, heads:heads + kvh], rows[:, heads + kvh:]
    other, before = _copy(cache), rows.clone()
    say("kv_append of %d tokens, heads %d and %d" % (T, heads, kvh))
    want_q, want_k = cts.rotary(q, k, cos, sin, pos, sections=sections)
    cts.kv_write(other, want_k, v, slots)
    torch.cuda.synchronize()
    with torch.cuda.stream(torch.cuda.Stream()):
        cts.kv_append(cache, q, k, v, slots, cos, sin, pos, sections=sections, q_out=q, k_out=k)
    torch.cuda.synchronize()
    assert torch.equal(k, want_k) and torch.equal(v, before[:, heads + kvh:]) and _same(cache, other)
    assert not heads or torch.equal(q, want_q)
