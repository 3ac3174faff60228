"""A verified tree of drafts from end to end: stored, attended to, cut back to what was accepted, and decoded from,
beside the same tokens decoded one after another; the decoder block with drafts, step by step against the oracle."""
import re

import numpy as np
import pytest
import torch

import paper_2407_00066_amd as cts
from oracle import block as ob
from paper_2407_00066_amd import decoder

from _block_helpers import ROUND, TORCH, assert_within, f64, to_host
from _draft_helpers import WEIGHTS, drafted, i32
from _gpu_helpers import say

pytestmark = pytest.mark.gpu


def _branch(parents, leaf):
    path = []
    while leaf >= 0:
        path.insert(0, leaf)
        leaf = parents[leaf]
    return path


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d,heads,kvh", [(64, 4, 2), (128, 8, 2), (256, 2, 1)])
def test_a_verified_tree_is_a_decoded_chain(d, heads, kvh, dtype):
    rng = np.random.default_rng(d)
    g = torch.Generator(device="cuda")
    g.manual_seed(d)
    page, past, n = 16, [37, 0, 200], [11, 4, 40]
    cos, sin = decoder.rotary_table(300, d)
    trees = [drafted(rng, m) for m in n]
    paths = [_branch(t[0], m - 1 - b) for b, (t, m) in enumerate(zip(trees, n))]
    need = [-(-(a + b) // page) for a, b in zip(past, n)]
    tables = [list(range(sum(need[:b]), sum(need[:b + 1]))) for b in range(3)]
    cols = max(need)
    table = i32(np.array([t + [0] * (cols - len(t)) for t in tables], np.int32))
    slot = lambda b, t: tables[b][t // page] * page + t % page
    new = lambda T, h: torch.randn(T, h, d, generator=g, device="cuda").to(TORCH[dtype])
    a, c = (cts.kv_cache(sum(need), page, kvh, d) for _ in range(2))
    # the prompts into both
    k, v = new(sum(past), kvh), new(sum(past), kvh)
    at = torch.tensor([slot(b, t) for b in range(3) for t in range(past[b])], device="cuda")
    pos = i32(np.array([t for b in range(3) for t in range(past[b])], np.int32))
    for cache in (a, c):
        assert cts.kv_append(cache, None, k, v, at, cos, sin, pos) is None
    # the drafts in one step
    T = sum(n)
    q, k, v = new(T, heads), new(T, kvh), new(T, kvh)
    start = np.concatenate(([0], np.cumsum(n)))
    mask = np.zeros((T, 2), np.uint32)
    depth = []
    for b in range(3):
        seen, dep = decoder.draft_tree(trees[b][0])
        assert dep == trees[b][1]
        depth += [past[b] + x for x in dep]
        for i, m in enumerate(seen):
            mask[start[b] + i] = [m & 0xffffffff, m >> 32]
    at = torch.tensor([slot(b, past[b] + i) for b in range(3) for i in range(n[b])], device="cuda")
    n_kv = i32(np.array([p + m for p, m in zip(past, n)], np.int32))
    say("a verified tree d=%d %s" % (d, dtype))
    tq = cts.kv_append(a, q, k, v, at, cos, sin, i32(np.array(depth, np.int32)))
    tree = cts.kv_tree_attention(tq, a, table, n_kv, i32(mask), q_start=i32(start.astype(np.int32)), max_q=max(n))
    most = max(map(len, paths))
    cts.kv_keep(a, table, n_kv, i32(start.astype(np.int32)), i32(np.array([p + [-1] * (most - len(p)) for p in paths], np.int32)),
                i32(np.array([len(p) for p in paths], np.int32)))
    # the accepted ones, as they come one after another
    rows = torch.tensor([start[b] + i for b in range(3) for i in paths[b]], device="cuda")
    m = [len(p) for p in paths]
    begin = np.concatenate(([0], np.cumsum(m))).astype(np.int32)
    at = torch.tensor([slot(b, past[b] + i) for b in range(3) for i in range(m[b])], device="cuda")
    pos = i32(np.array([past[b] + i for b in range(3) for i in range(m[b])], np.int32))
    cq = cts.kv_append(c, q[rows], k[rows], v[rows], at, cos, sin, pos)
    assert torch.equal(cq, tq[rows])
    length = i32(np.array([p + x for p, x in zip(past, m)], np.int32))
    chain = cts.kv_attention(cq, c, table, length, q_start=i32(begin), max_q=max(m))
    # each is within its own bound of the exact result
    want, mag, soft = ob.attention(f64(cq), to_host(c), table.cpu().numpy(), length.cpu().numpy(), begin, d ** -0.5)
    bound = 1.01 * (ROUND[dtype] * np.abs(want) + WEIGHTS[dtype] * mag + soft) + 1e-30
    assert_within(tree[rows], want, bound, "tree")
    assert_within(chain, want, bound, "chain")
    # the caches hold the same tokens, and the next token sees the same
    at = torch.tensor([slot(b, t) for b in range(3) for t in range(past[b] + m[b])], device="cuda")
    for x, y in zip(cts.kv_read(a, at, dtype=torch.float32), cts.kv_read(c, at, dtype=torch.float32)):
        assert torch.equal(x, y)
    q1 = new(3, heads)
    assert torch.equal(cts.kv_attention(q1, a, table, length), cts.kv_attention(q1, c, table, length))


def test_block_with_drafts():
    """DecoderBlock.forward on a Batch with parents: positions, cache and attention against the oracle."""
    D, heads, kv, hd, ff, n, K, r, page = 256, 4, 2, 64, 320, 9, 3, 16, 16
    w = decoder.random_weights(D, heads, kv, hd, ff, n, K, r, seed=4)
    cos, sin = decoder.rotary_table(200, hd)
    cache = cts.kv_cache(24, page, kv, hd)
    blk = decoder.DecoderBlock(w, heads, kv, hd, cache, cos, sin)
    cluster_of = torch.arange(n, dtype=torch.int32, device="cuda") % K
    tables = [[5, 0, 9, 14], [1, 2, 3, 4], [20, 21, 22, 23]]
    make = lambda *a, **kw: decoder.Batch([7, 0, 4], cluster_of, n, K, *a, tables, page, **kw)
    torch.manual_seed(0)
    new = lambda batch: torch.randn(batch.T, D, device="cuda").bfloat16()
    prompt = make([33, 5, 17], [33, 5, 17])
    blk.forward(new(prompt), None, prompt)
    parents = [[-1, 0, 0, 1, 2, 2, -1], None, [-1, -1, 0]]
    counts, lens = [7, 4, 3], [40, 9, 20]
    batch = make(counts, lens, parents=parents)
    assert batch.positions.tolist() == [33, 34, 34, 35, 35, 35, 33, 5, 6, 7, 8, 17, 17, 18]
    before = tuple(a.copy() for a in to_host(cache))
    keep, plain = {}, {}
    h, y = new(batch), new(batch)
    say("decoder block with drafts")
    h2, y2 = blk.forward(h, y, batch, keep)
    torch.cuda.synchronize()
    qkv, pos = f64(keep["qkv"]), batch.positions.cpu().numpy()
    for name, lo, count in (("q", 0, heads), ("k", heads, kv)):
        x = qkv[:, lo * hd:(lo + count) * hd].reshape(-1, count, hd)
        want, mag = ob.rotary(x, f64(cos), f64(sin), pos[None], [hd // 2])
        assert_within(keep[name], want, 1.01 * ROUND["bf16"] * np.abs(want) + 2.0 ** -22 * mag, name)
    ob.write(before, f64(keep["k"]), f64(keep["v"]), batch.slots.cpu().numpy())
    assert all(np.array_equal(a, b) for a, b in zip(to_host(cache), before))
    start = np.concatenate(([0], np.cumsum(counts)))
    mask = batch.mask.cpu().numpy().view(np.uint32)
    assert mask[:, 0].tolist() == [1, 3, 5, 0b1011, 0b10101, 0b100101, 64, 1, 3, 7, 15, 1, 2, 5]
    want, mag, soft = ob.tree_attention(f64(keep["q"]), before, batch.table.cpu().numpy(), lens, start, mask, hd ** -0.5)
    assert_within(keep["a"], want, 1.01 * (ROUND["bf16"] * np.abs(want) + 2.0 ** -8 * mag + soft) + 1e-30, "attention")
    # the values between the steps are not needed for the result
    h3, y3 = blk.forward(h, y, batch)
    assert torch.equal(h2, h3) and torch.equal(y2, y3)
    path, n_path = [[0, 2, 5], [0, 1, -1], [-1, -1, -1]], [3, 2, 0]
    blk.keep_accepted(batch, i32(np.array(path, np.int32)), i32(np.array(n_path, np.int32)))
    torch.cuda.synchronize()
    ob.keep(before, np.array(tables), lens, start, np.array(path), n_path)
    assert all(np.array_equal(a, b) for a, b in zip(to_host(cache), before))


@pytest.mark.parametrize("counts,parents", [([1], [[0]]), ([3], [[-1, 2, 0]]), ([2], [[-1, 1]]), ([1], [[-2]]), ([3], [[-1, 0]]),
                                            ([1], [[-1], [-1]]), ([1, 1], [None]), ([600], [range(-1, 599)]), ([513], [None])])
def test_batch_refuses_what_is_no_tree(counts, parents):
    cluster_of = torch.zeros(2, dtype=torch.int32, device="cuda")
    with pytest.raises(ValueError):
        decoder.Batch([0] * len(counts), cluster_of, 2, 1, counts, [600] * len(counts), [range(40)] * len(counts), 16, parents=parents)


def test_command_times_drafts(capsys):
    say("decoder command with drafts")
    decoder.main(["--requests", "2", "--context", "33", "--layers", "1", "--steps", "2", "--drafts", "5"])
    out = capsys.readouterr().out
    found = re.search(r"drafts: 2 requests, 5 each, 1 layers: ([0-9.]+) ms a step, ([0-9.]+) with the batch's preparation", out)
    assert found and 0 < float(found[1]) < float(found[2])
    decoder.main(["--requests", "1", "--context", "3", "--layers", "1", "--steps", "1", "--drafts", "0"])
    assert "drafts" not in capsys.readouterr().out
    for bad in ("-1", "513"):
        with pytest.raises(SystemExit):
            decoder.main(["--drafts", bad])


def test_a_captured_step():
    """Stored, attended to and cut back in one graph: replays with other tokens, lengths, masks and paths equal eager
    calls, with eager work between."""
    rng = np.random.default_rng(3)
    page, cols, n, kvh, heads, d = 16, 40, [12, 7, 30], 2, 8, 128
    T, start = sum(n), i32(np.concatenate(([0], np.cumsum(n))).astype(np.int32))
    table = np.arange(3 * cols, dtype=np.int32).reshape(3, cols)
    cos, sin = decoder.rotary_table(700, d)
    cache, other = (cts.kv_cache(3 * cols, page, kvh, d) for _ in range(2))
    q, k, v = (torch.zeros(T, h, d, dtype=torch.bfloat16, device="cuda") for h in (heads, kvh, kvh))
    slots, pos = torch.zeros(T, dtype=torch.int64, device="cuda"), torch.zeros(T, dtype=torch.int32, device="cuda")
    mask, n_kv = torch.zeros(T, 1, dtype=torch.int32, device="cuda"), i32(np.array(n, np.int32))
    path, n_path = torch.zeros(3, 5, dtype=torch.int32, device="cuda"), torch.zeros(3, dtype=torch.int32, device="cuda")
    tables, out = i32(table), torch.empty_like(q)
    ws = torch.empty(cts.kv_tree_attention_workspace_size(q, cache, 3, 30, cols * page), dtype=torch.uint8, device="cuda")

    def step(kv, o):
        turned = cts.kv_append(kv, q, k, v, slots, cos, sin, pos)
        cts.kv_tree_attention(turned, kv, tables, n_kv, mask, q_start=start, max_q=30, out=o, workspace=ws)
        cts.kv_keep(kv, tables, n_kv, start, path, n_path)

    for a in (cache.k_codes, cache.v_codes):
        a.random_(0, 256)
    for a in (cache.k_scales, cache.v_scales):
        a.random_(122, 128)
    step(cache, out)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step(cache, out)
    for i in range(3):
        past = rng.integers(0, 600, 3)
        at = [[table[b][t // page] * page + t % page for t in range(past[b], past[b] + n[b])] for b in range(3)]
        slots.copy_(torch.tensor(sum(at, [])))
        n_kv.copy_(torch.from_numpy((past + n).astype(np.int32)))
        pos.copy_(torch.from_numpy(np.concatenate([past[b] + np.arange(n[b]) // 2 for b in range(3)]).astype(np.int32)))
        mask.copy_(torch.from_numpy(rng.integers(0, 2 ** 32, (T, 1), dtype=np.uint32).view(np.int32)))
        path.copy_(torch.from_numpy(rng.integers(0, 7, (3, 5)).astype(np.int32)))
        n_path.copy_(torch.from_numpy(rng.integers(0, 6, 3).astype(np.int32)))
        for t in (q, k, v):
            t.copy_(torch.randn(t.shape, device="cuda"))
        for a, b in zip((cache.k_codes, cache.k_scales, cache.v_codes, cache.v_scales),
                        (other.k_codes, other.k_scales, other.v_codes, other.v_scales)):
            b.copy_(a)
        say("a captured step, replay %d" % i)
        g.replay()
        torch.cuda.synchronize()
        want = torch.empty_like(q)
        step(other, want)
        torch.cuda.synchronize()
        assert torch.equal(out, want)
        assert all(np.array_equal(a, b) for a, b in zip(to_host(cache), to_host(other)))
