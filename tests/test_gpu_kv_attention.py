"""cts_kv_attention against the oracle on the same cache.

Bound of an element's error: half a step of the output type; bf16 also rounds
every weight once (2^-8 of sum w |v|), f32 keeps 24 bits of it (three parts:
2^-22 allowed); and what fp32 sums leave (the oracle's third result)."""
import numpy as np
import pytest
import torch

import paper_2407_00066_amd as cts
from oracle import block as ob

from _block_helpers import ROUND, TORCH, assert_within, to_device, values
from _gpu_helpers import say

pytestmark = pytest.mark.gpu

WEIGHTS = {"bf16": 2.0 ** -8, "f32": 2.0 ** -22}


def make(n_q, n_kv, heads, kvh, d, page, dtype="bf16", seed=0, spare=2, fill=None, big=1.0):
    """A filled cache (every slot of every page, the unused ones too), a table of pages in no order, queries."""
    rng = np.random.default_rng(seed)
    need = [-(-n // page) for n in n_kv]
    pages = sum(need) + spare
    cols = max(need + [1])
    order = rng.permutation(pages)
    table, used = np.zeros((len(n_kv), cols), np.int32), 0
    for b, n in enumerate(need):
        table[b, :n] = order[used:used + n]
        used += n
    cache = ob.empty_cache(pages, page, kvh, d)
    for a in (cache[0], cache[2]):
        a[...] = rng.integers(0, 256, a.shape)
    for a in (cache[1], cache[3]):
        a[...] = rng.integers(122, 128, a.shape)
    q_start = np.concatenate(([0], np.cumsum(n_q))).astype(np.int32)
    q64, q = values(rng, (q_start[-1], heads, d), dtype, big)
    return {"cache": cache, "table": table, "n_kv": np.array(n_kv, np.int32), "q_start": q_start, "q64": q64, "q": q,
            "heads": heads, "dtype": dtype, "max_q": max(list(n_q) + [1]), "d": d}


def call(c, window=0, **kw):
    cache = to_device(c["cache"])
    out = cts.kv_attention(kw.pop("q", c["q"]), cache, torch.from_numpy(c["table"]).cuda(), torch.from_numpy(c["n_kv"]).cuda(),
                           q_start=torch.from_numpy(c["q_start"]).cuda(), max_q=c["max_q"], window=window, **kw)
    torch.cuda.synchronize()
    return out


def check(c, window=0, scale=None, **kw):
    say("kv_attention %s q=%s kv=%s heads=%d d=%d window=%d" % (c["dtype"], np.diff(c["q_start"]).tolist()[:8],
                                                                c["n_kv"].tolist()[:8], c["heads"], c["d"], window))
    out = call(c, window, scale=scale, **kw)
    want, mag, soft = ob.attention(c["q64"], c["cache"], c["table"], c["n_kv"], c["q_start"],
                                   c["d"] ** -0.5 if scale is None else scale, window)
    r = ROUND[c["dtype"]]
    assert_within(out, want, 1.01 * (r * np.abs(want) + WEIGHTS[c["dtype"]] * mag + soft) + 1e-30, "kv_attention")
    return out


# lengths around every step and tile, one token a sequence
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d,page", [(64, 16), (128, 16), (256, 32), (128, 128)])
def test_decode_lengths(d, page, dtype):
    n_kv = [0, 1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 255, 300, 511]
    check(make([1] * len(n_kv), n_kv, 8, 2, d, page, dtype, seed=d + page))


# query heads of a key/value head: 1, odd counts, more than a tile's 16 rows
@pytest.mark.parametrize("heads,kvh", [(1, 1), (3, 3), (5, 1), (12, 4), (16, 1), (17, 1), (40, 1), (64, 2), (71, 1)])
def test_head_groups(heads, kvh):
    check(make([1, 1, 1], [77, 1, 130], heads, kvh, 128, 16, seed=heads))
    check(make([3, 1, 6], [77, 1, 130], heads, kvh, 64, 16, seed=heads + 1))


# several queries a sequence: drafts, prompts without a past, chunks after one
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n_q,n_kv,heads,kvh,d", [
    ([5, 1, 4], [40, 9, 4], 8, 2, 128), ([16, 17, 33], [16, 17, 33], 4, 4, 64), ([65, 64, 1, 0, 3], [65, 200, 7, 5, 500], 8, 2, 128),
    ([130], [400], 6, 2, 128), ([128, 127], [128, 300], 4, 1, 64), ([20, 70], [33, 70], 4, 2, 256),
    ([300, 1, 257], [300, 1000, 257], 4, 1, 128), ([513], [513], 1, 1, 128), ([260], [900], 2, 1, 64)])
def test_prompts(n_q, n_kv, heads, kvh, d, dtype):
    check(make(n_q, n_kv, heads, kvh, d, 16, dtype, seed=sum(n_q) + d))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("window", [1, 2, 31, 32, 33, 100, 5000])
def test_window(window, dtype):
    check(make([1, 7, 40, 1, 150], [300, 64, 90, 33, 420], 4, 2, 64, 16, dtype, seed=window), window=window)
    check(make([1, 1, 1], [300, 1, 33], 4, 2, 128, 16, dtype, seed=window), window=window)


def test_rows_that_see_nothing():
    """More queries than cached tokens: the first ones see nothing and give zeros; so does an empty cache."""
    c = make([5, 3, 1, 200], [2, 0, 0, 90], 8, 2, 128, 16, seed=3)
    out = check(c)
    assert not out[:3].any() and not out[5:9].any() and not out[9:9 + 110].any() and out[9 + 110:].any()


def test_long_sequences_in_pieces():
    """One request over a long context (the work is split along it and joined), beside short ones."""
    check(make([1], [3001], 4, 1, 128, 16, seed=8))
    check(make([1, 1, 2], [2500, 40, 3], 8, 2, 64, 64, seed=9))
    check(make([1, 1], [1700, 900], 2, 2, 256, 16, "f32", seed=10))


# a bound far above the lengths: the steps are dealt out over the whole card, runs begin and
# end inside sequences, cover several of them, or a few sequences are cut into pieces
@pytest.mark.parametrize("window", [0, 45])
@pytest.mark.parametrize("d,dtype", [(64, "bf16"), (128, "bf16"), (256, "bf16"), (128, "f32"), (64, "f32")])
@pytest.mark.parametrize("B,kvh,top", [(3, 2, 2600), (7, 3, 1500), (90, 1, 300), (40, 4, 700), (1, 1, 4000)])
def test_equal_runs(B, kvh, top, d, dtype, window):
    rng = np.random.default_rng(B + d)
    n_kv = rng.integers(1, top, B)
    n_kv[0], n_kv[-1], n_kv[B // 2] = top, max(1, top - 77), 3 if B > 1 else top
    n_q = np.minimum(rng.integers(1, 4, B), n_kv)
    if B > 4:                                                        # nothing cached, no rows, many rows
        n_kv[2], n_q[3], n_q[4], n_kv[4] = 0, 0, 40, 200
    check(make(n_q.tolist(), n_kv.tolist(), 2 * kvh, kvh, d, 16, dtype, seed=B + d), window=window, max_kv=10 ** 6)


# one to two workgroups for every compute unit: they take the sequences in the order of their lengths
@pytest.mark.parametrize("B,kvh,d", [(64, 8, 64), (33, 8, 128), (65, 4, 64), (128, 3, 64), (2, 200, 64), (40, 12, 64), (1, 300, 64), (128, 4, 64)])
def test_sequences_in_order_of_length(B, kvh, d):
    rng = np.random.default_rng(B)
    n_kv = rng.integers(0, 150, B)
    n_kv[1::5] = 64                                                  # equal ones among them
    check(make([1] * B, n_kv.tolist(), kvh, kvh, d, 16, seed=B), max_kv=2000)
    n_q = np.minimum(rng.integers(0, 4, B), n_kv)
    check(make(n_q.tolist(), n_kv.tolist(), 9 * kvh, kvh, d, 16, seed=B + 1), max_kv=2000)
    n_kv[:] = 1
    check(make([1] * B, n_kv.tolist(), kvh, kvh, d, 16, seed=B + 2), max_kv=2000)


def test_more_steps_than_runs_of_one():
    """Runs of several steps a wave, of unequal sequences; heads that leave a compute unit idle."""
    check(make([1, 1, 1], [20011, 9000, 33], 5, 5, 64, 32, seed=15))
    check(make([2, 1], [17000, 31], 3, 1, 128, 64, seed=16))
    check(make([1] * 66, [130 * i + 7 for i in range(66)], 1, 1, 128, 16, seed=17), max_kv=10 ** 6)


def test_max_kv_and_wider_tables():
    """max_kv only has to bound the lengths: a loose and a tight one, and a wider table, agree with the oracle."""
    c = make([1, 2], [333, 200], 8, 2, 128, 16, seed=12)
    a = check(c, max_kv=333)
    wide = np.full((2, 4096), 2 ** 30, np.int32)                    # columns past the lengths are never used
    wide[:, :c["table"].shape[1]] = c["table"]
    c["table"] = wide
    b = check(c, max_kv=10 ** 6)
    assert_within(a, b.double().cpu().numpy(), 0.02, "two splits")


def test_scale_and_large_scores():
    """Scores of several hundred: the running maximum carries them."""
    c = make([1, 9], [500, 300], 8, 2, 128, 16, seed=13, big=30.0)
    check(c, scale=0.5)
    check(make([1, 9], [500, 300], 8, 2, 128, 16, seed=14), scale=1e-3)


def _poison(c, b, tokens, what):
    """NaN scales on tokens' keys and values."""
    page = c["cache"][0].shape[2]
    for t in tokens:
        p, o = int(c["table"][b][t // page]), t % page
        if "k" in what:
            c["cache"][1][p, :, o] = 255
        if "v" in what:
            c["cache"][3][p, :, o // 4, :, o % 4] = 255


@pytest.mark.parametrize("d,n_q,window", [(128, 40, 0), (64, 40, 0), (256, 9, 0), (128, 40, 20), (128, 300, 0),
                                          (64, 300, 64)])
def test_nan_behind_the_mask(d, n_q, window):
    """NaN keys and values at tokens that only later queries see, and past the
    end: the rows that do not see them come out as if they were not there."""
    L = n_q + 25
    c = make([n_q], [L], 4, 2, d, 32, seed=d + n_q)
    cut = L - n_q // 3
    clean = ob.attention(c["q64"], c["cache"], c["table"], c["n_kv"], c["q_start"], d ** -0.5, window)
    _poison(c, 0, [cut], "kv")
    _poison(c, 0, [cut + 2], "v")
    page = 32
    last = int(c["table"][0][(L - 1) // page])
    c["cache"][1][last, :, (L - 1) % page + 1:] = 255               # what lies past the end in its page
    for o in range((L - 1) % page + 1, page):
        c["cache"][3][last, :, o // 4, :, o % 4] = 255
    out = check(c, window)
    rows = cut - (L - n_q)
    assert not torch.isnan(out[:rows]).any() and torch.isnan(out[rows]).any()
    r = ROUND["bf16"]
    want, mag, soft = (a[:rows] for a in clean)
    assert_within(out[:rows], want, 1.01 * (r * np.abs(want) + 2.0 ** -8 * mag + soft), "rows before the NaN")


def test_nan_in_one_block_of_a_value():
    """A NaN block of a seen value makes its 32 elements NaN and no others."""
    c = make([1, 12], [50, 44], 4, 2, 128, 16, seed=21)
    p, o = int(c["table"][1][2]), 3                                  # token 35 of sequence 1
    c["cache"][3][p, 1, o // 4, 2, o % 4] = 255
    out = check(c)
    assert torch.isnan(out[1 + 3:, 2:, 64:96]).all() and not torch.isnan(out[:, :2]).any()


def test_infinite_queries_and_zero_scores():
    c = make([1, 1, 1], [40, 33, 9], 4, 2, 128, 16, seed=22)
    q = c["q"].clone()
    q[1] = 0                                                          # all weights equal
    c["q64"][1] = 0
    c["q"] = q
    check(c)
    q = q.clone()
    q[2, 0, 5] = float("inf")
    out = call(c, q=q)
    assert torch.isnan(out[2, 0]).all() and not torch.isnan(out[2, 1:]).any() and not torch.isnan(out[:2]).any()


@pytest.mark.parametrize("n_q", [1, 30, 300])
def test_pages_outside_the_cache_read_as_nan(n_q):
    """A page number outside the cache never reads outside it: its tokens are NaN."""
    c = make([n_q, n_q], [n_q + 70, n_q + 70], 4, 2, 128, 16, seed=23)
    c["table"][1, 1] = 2 ** 30
    c["table"][1, 2] = -5
    out = call(c)
    assert torch.isnan(out[n_q:]).all() and not torch.isnan(out[:n_q]).any()


def test_lengths_and_starts_are_clamped():
    """Lengths past max_kv and starts out of order: nothing outside is touched."""
    c = make([1, 1], [40, 40], 4, 2, 64, 16, seed=24)
    c["n_kv"] = np.array([10 ** 9, -7], np.int32)
    c["q_start"] = np.array([0, 1, -3], np.int32)
    guard = torch.full((4, 4, 64), 7.0, dtype=torch.bfloat16, device="cuda")
    call(c, out=guard[1:3], max_kv=40)
    assert bool((guard[0] == 7).all()) and bool((guard[2:] == 7).all())


def test_strides_and_untouched_rows():
    """q from packed rows, out into wider ones; rows of no sequence keep what they held."""
    c = make([2, 3], [60, 50], 4, 2, 128, 16, seed=25)
    plain = call(c)
    packed = torch.full((6, 10 * 128), 3.0, dtype=torch.bfloat16, device="cuda")
    packed[:5, 128:640] = c["q"].flatten(1)
    out = torch.full((6, 6, 128), 5.0, dtype=torch.bfloat16, device="cuda")
    call(c, q=packed[:, 128:640].unflatten(1, (4, 128)), out=out[:, 1:5])
    assert torch.equal(out[:5, 1:5], plain) and bool((out[5] == 5).all()) and bool((out[:, [0, 5]] == 5).all())


def test_none_starts_and_zero_rows():
    c = make([1] * 5, [9, 100, 1, 64, 300], 8, 8, 64, 16, seed=26)
    cache, table, n_kv = to_device(c["cache"]), torch.from_numpy(c["table"]).cuda(), torch.from_numpy(c["n_kv"]).cuda()
    assert torch.equal(cts.kv_attention(c["q"], cache, table, n_kv), call(c))
    assert cts.kv_attention(c["q"][:0], cache, table[:0], n_kv[:0]).shape == (0, 8, 64)


def test_same_bits_every_time_and_on_another_stream():
    c = make([1, 30, 400], [2000, 100, 400], 8, 2, 128, 16, seed=27)
    a = call(c)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        b = call(c)
    side.synchronize()
    assert torch.equal(a, b) and torch.equal(a, call(c))


def test_workspace_serves_smaller_batches():
    c = make([1, 30, 400], [2000, 100, 400], 8, 2, 128, 16, seed=28)
    need = cts.kv_attention_workspace_size(c["q"], to_device(c["cache"]), 3, 400, 2000)
    ws = torch.full((need + 256,), 255, dtype=torch.uint8, device="cuda")
    check(c, workspace=ws[:need], max_kv=2000)
    check(make([1, 3], [900, 100], 8, 2, 128, 16, seed=29), workspace=ws[:need], max_kv=1000)
    assert bool((ws[need:] == 255).all())


def test_graph_replays():
    """Captured once, replayed with new lengths, queries and cache contents; eager work between."""
    c = make([1] * 6, [5, 700, 64, 1500, 33, 1], 8, 2, 128, 16, seed=30)
    cache, table, n_kv = to_device(c["cache"]), torch.from_numpy(c["table"]).cuda(), torch.from_numpy(c["n_kv"]).cuda()
    q = c["q"].clone()
    new = torch.randn(6, 2, 2, 128, device="cuda").bfloat16()
    slots = table.long()[torch.arange(6), (n_kv.long() - 1) // 16] * 16 + (n_kv.long() - 1) % 16
    out = torch.empty_like(q)

    def step(o):
        cts.kv_write(cache, new[:, 0], new[:, 1], slots)
        return cts.kv_attention(q, cache, table, n_kv, max_kv=1500, out=o)
    step(out)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step(out)
    for rep in range(4):
        q.normal_()
        new.normal_()
        n_kv.sub_(1 if rep == 2 else 0).clamp_(min=0)
        out.fill_(float("nan"))
        say("graph replay %d" % rep)
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, step(torch.empty_like(q)))


def test_cache_past_32_bits():
    """Pages whose bytes lie past 2^32."""
    pages, page, heads, d = 2200, 1024, 32, 128                     # 4.6 GB of key codes
    cache = cts.kv_cache(pages, page, heads, d)
    table = torch.tensor([[pages - 1], [0]], dtype=torch.int32, device="cuda")
    rng = np.random.default_rng(31)
    k64, k = values(rng, (3, heads, d), "bf16")
    slots = (pages - 1) * page + torch.arange(3, device="cuda")
    cts.kv_write(cache, k, k, slots)
    q64, q = values(rng, (2, heads, d), "bf16")
    say("kv_attention past 32 bits")
    out = cts.kv_attention(q, cache, table, torch.tensor([3, 1], dtype=torch.int32, device="cuda"))
    K = ob.dequantize(*ob.quantize(k64))
    s = np.einsum("hd,thd->ht", q64[0], K) * d ** -0.5
    w = np.exp(s - s.max(1, keepdims=True))
    w /= w.sum(1, keepdims=True)
    want = np.einsum("ht,thd->hd", w, K)
    mag = np.einsum("ht,thd->hd", w, np.abs(K))
    assert_within(out[0], want, 2.0 ** -8 * 1.02 * (np.abs(want) + mag), "past 32 bits")
    assert not out[1].any()


def test_types_are_checked():
    assert TORCH["bf16"] == torch.bfloat16
    c = make([1], [5], 4, 2, 64, 16)
    cache, table, n_kv = to_device(c["cache"]), torch.from_numpy(c["table"]).cuda(), torch.from_numpy(c["n_kv"]).cuda()
    with pytest.raises(TypeError):
        cts.kv_attention(c["q"].half(), cache, table, n_kv)
    with pytest.raises(TypeError):
        cts.kv_attention(c["q"], cache, table.long(), n_kv)
    with pytest.raises(ValueError):
        cts.kv_attention(c["q"], cache, table, n_kv[:0])
    with pytest.raises(cts.CtsError):
        cts.kv_attention(c["q"], cache, table, n_kv, max_q=2)
    with pytest.raises(cts.CtsError):
        cts.kv_attention(c["q"], cache, table, n_kv, workspace=torch.empty(16, dtype=torch.uint8, device="cuda"))
