"""cts_kv_tree_attention under every way its work is dealt out, which cts_kv_tree_attention_plan names: tiles of
16, 32 and 64 rows, whole, by their work, and cut along their tokens (wide tables make loose bounds)."""
import numpy as np
import pytest
import torch

import paper_2407_00066_amd as cts

from _block_helpers import to_device
from _draft_helpers import call, check, i32, make
from _gpu_helpers import say

pytestmark = pytest.mark.gpu


def _widen(c, cols):
    """Columns past the sequences' pages, which are never used."""
    wide = np.full((c["table"].shape[0], cols), 2 ** 30, np.int32)
    wide[:, :c["table"].shape[1]] = c["table"]
    c["table"] = wide
    return c


def _plan(c, window=0):
    cache = cts.kv_cache(1, c["cache"][0].shape[2], c["cache"][0].shape[1], c["d"])
    table = torch.from_numpy(c["table"])
    return cts.kv_tree_attention_plan(c["q"], cache, table, c["max_q"], c["table"].shape[1] * c["cache"][0].shape[2], window)


# few tiles cut into many pieces, of every number of rows; lengths from nothing to many steps
@pytest.mark.parametrize("window", [0, 70])
@pytest.mark.parametrize("d,heads,kvh,dtype,rows", [(64, 4, 1, "bf16", 64), (128, 4, 1, "bf16", 64), (128, 2, 1, "bf16", 32),
                                                    (256, 4, 1, "bf16", 32), (64, 4, 1, "f32", 32), (128, 4, 1, "f32", 32),
                                                    (256, 1, 1, "f32", 16), (128, 16, 16, "bf16", 16)])
def test_few_tiles_cut(d, heads, kvh, dtype, rows, window):
    n_q, n_past = [16, 3, 9, 14, 1, 0, 5], [2500, 1, 700, 0, 2047, 90, 33]
    if rows == 64:
        n_q[2] = 37                                              # several tiles of a sequence
    c = _widen(make(n_q, n_past, heads, kvh, d, 16, dtype, seed=d + heads + window), 8192 if not window else 200)
    got = _plan(c, window)
    assert got[1] == ("cut" if not window else "whole") and (window or got[0] == rows), got
    check(c, window)


def test_few_tiles_cut_under_a_window():
    c = _widen(make([16, 5, 9], [3500, 40, 2600], 4, 1, 64, 16, seed=3), 8192)
    assert _plan(c, 2100)[1] == "cut"
    check(c, 2100)


# more than 64 tiles, found without their order; more tiles than workgroups run at a time
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("B,kvh,top", [(90, 1, 500), (70, 8, 300), (40, 16, 260), (300, 2, 120)])
def test_many_tiles_cut(B, kvh, top, d):
    rng = np.random.default_rng(B + d)
    n_q, n_past = rng.integers(0, 5, B), rng.integers(0, top, B)
    n_past[B // 2], n_past[3], n_q[3], n_q[B // 2] = 2900, 0, 0, 3
    c = _widen(make(n_q.tolist(), n_past.tolist(), 2 * kvh, kvh, d, 16, seed=B), 700)
    assert _plan(c)[1] == "cut"
    check(c)


# more workgroups than compute units take their tiles by work
@pytest.mark.parametrize("B,kvh,heads,d,dtype", [(40, 8, 8, 64, "bf16"), (64, 8, 32, 128, "bf16"), (200, 2, 4, 64, "bf16"),
                                                 (256, 2, 2, 64, "f32"), (65, 4, 8, 256, "bf16")])
def test_tiles_by_work(B, kvh, heads, d, dtype):
    rng = np.random.default_rng(B)
    n_q, n_past = rng.integers(0, 7, B), rng.integers(0, 180, B)
    n_q[1::7], n_past[1::7] = 4, 60                              # equal ones among them
    c = make(n_q.tolist(), n_past.tolist(), heads, kvh, d, 16, dtype, seed=B)
    assert _plan(c)[1] == "by work"
    check(c)


def test_more_tiles_than_are_ordered():
    c = make([2] * 300, [i % 40 for i in range(300)], 2, 1, 64, 16, seed=9)
    assert _plan(c)[1] == "whole"
    check(c)


@pytest.mark.parametrize("rows,n,B", [(16, 4, 3), (32, 8, 200), (64, 16, 200)])
def test_rows_of_a_tile(rows, n, B):
    """Tiles of as many rows as a sequence has, but of 16 where there is little work."""
    cache, q = cts.kv_cache(1, 16, 8, 128), torch.zeros(n * B, 32, 128, dtype=torch.bfloat16, device="cuda")
    table = torch.zeros(B, 60, dtype=torch.int32)
    assert cts.kv_tree_attention_plan(q, cache, table, n, 900)[0] == rows
    assert cts.kv_tree_attention_plan(q[:16], cache, table[:1], 16, 900)[0] == 16


def test_counted_tokens_of_cut_tiles():
    """Queries of zero weigh what they see alike: with the last draft worth 2 and all else 1, the result is 1 + 1 / seen."""
    for d, kvh, dtype in ((128, 2, "f32"), (64, 1, "bf16")):
        n_q, n_past = [13, 40, 2], [2311, 999, 64]
        c = _widen(make(n_q, n_past, 2 * kvh, kvh, d, 16, dtype, seed=d), 8192)
        c["q"].zero_()
        c["cache"][2][...], c["cache"][3][...] = 0x22, 127       # every value is 1
        for b, m in enumerate(n_q):
            t = int(c["n_kv"][b]) - 1
            c["cache"][2][int(c["table"][b][t // 16]), :, t % 16 // 4, :, t % 4] = 0x44
        assert _plan(c)[1] == "cut"
        say("kv_tree_attention counting, d=%d %s" % (d, dtype))
        out = call(c).double().cpu().numpy()
        for b, (m, past) in enumerate(zip(n_q, n_past)):
            for j in range(m):
                row = int(c["q_start"][b]) + j
                bits = [i for i in range(m) if int(c["mask"][row][i // 32]) >> (i % 32) & 1]
                want = 1.0 + (m - 1 in bits) / (past + len(bits))
                # (half a step of the output; fp32 sums of equal weights up to 2400, and a division)
                bound = {"f32": 2.0 ** -20, "bf16": 1.01 * 2.0 ** -8}[dtype]
                assert np.abs(out[row] - want).max() <= bound * want, (b, j)


def test_pages_past_32_bits():
    """Pages whose bytes lie past 2^32."""
    n, page, kvh, d = 40000, 1024, 2, 256
    cache = cts.kv_cache(n, page, kvh, d)
    small = cts.kv_cache(3, page, kvh, d)
    far, near = [39999, 17000, 25001], [0, 1, 2]
    for a, b in ((cache.k_codes, small.k_codes), (cache.v_codes, small.v_codes)):
        b.random_(0, 256)
        for x, y in zip(far, near):
            a[x] = b[y]
    for a, b in ((cache.k_scales, small.k_scales), (cache.v_scales, small.v_scales)):
        b.random_(122, 128)
        for x, y in zip(far, near):
            a[x] = b[y]
    c = make([30], [2500], 4, 2, 256, 16, seed=5)
    args = [i32(c["n_kv"]), i32(c["mask"])]
    say("kv_tree_attention past 32 bits")
    t = lambda v: torch.tensor([v], dtype=torch.int32, device="cuda")
    a = cts.kv_tree_attention(c["q"], cache, t(far), *args, q_start=i32(c["q_start"]))
    b = cts.kv_tree_attention(c["q"], small, t(near), *args, q_start=i32(c["q_start"]))
    assert torch.equal(a, b)


def test_captured_and_replayed_with_other_lengths():
    """A captured call finds its work in the arrays: replays with other lengths, masks and queries equal eager calls, with
    eager work between; two graphs use one workspace in turn."""
    c = _widen(make([12, 16, 5, 30], [900, 40, 2500, 300], 4, 2, 64, 16, seed=41), 8192)
    cache, table, start = to_device(c["cache"]), i32(c["table"]), i32(c["q_start"])
    q, mask, n_kv = c["q"].clone(), i32(c["mask"]), i32(c["n_kv"])
    need = cts.kv_tree_attention_workspace_size(q, cache, 4, 30, 8192 * 16)
    ws = torch.empty(need, dtype=torch.uint8, device="cuda")
    outs = [torch.zeros_like(q) for _ in range(2)]
    run = lambda out: cts.kv_tree_attention(q, cache, table, n_kv, mask, q_start=start, max_q=30, out=out, workspace=ws)
    run(outs[0])
    torch.cuda.synchronize()
    graphs = []
    for o in outs:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            run(o)
        graphs.append(g)
    rng = np.random.default_rng(1)
    for i in range(4):
        n_kv.copy_(torch.from_numpy((c["n_kv"] - rng.integers(0, 40, 4)).clip(0).astype(np.int32)))
        mask.copy_(torch.from_numpy(rng.integers(0, 2 ** 32, c["mask"].shape, dtype=np.uint32).view(np.int32)))
        q.copy_(torch.randn_like(q.float()).bfloat16())
        for o, g in zip(outs, graphs):
            o.fill_(7)
            say("kv_tree_attention replay %d" % i)
            g.replay()
        torch.cuda.synchronize()
        want = run(None)
        torch.cuda.synchronize()
        assert torch.equal(outs[0], want) and torch.equal(outs[1], want)


def test_two_streams_at_once():
    c = make([16] * 6, [900, 40, 2000, 300, 5, 77], 8, 2, 128, 16, seed=43)
    cache = to_device(c["cache"])
    want = call(c, cache=cache)
    streams, outs = [torch.cuda.Stream() for _ in range(2)], []
    for s in streams:
        s.wait_stream(torch.cuda.current_stream())
    say("kv_tree_attention on two streams")
    args = [i32(a) for a in (c["table"], c["n_kv"], c["mask"], c["q_start"])]
    torch.cuda.synchronize()
    for _ in range(4):
        for s in streams:
            with torch.cuda.stream(s):
                outs.append(cts.kv_tree_attention(c["q"], cache, *args[:3], q_start=args[3], max_q=16))
    torch.cuda.synchronize()
    assert all(torch.equal(o, want) for o in outs)
