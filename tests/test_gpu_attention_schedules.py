"""cts_kv_attention under every way its work is dealt out, each asserted to be the one
that ran: whole tiles in the batch's order and by length, few tiles cut into runs
of their own, runs that go from tile to tile and head to head, prompts in pieces.

Two references, in 64 bits over the whole cache at once: attention itself (bounds
as in test_gpu_kv_attention.py), and counts.  With queries of zero every weight is
1: the output is the mean of the seen values.  Each token's value is 1 in one
element of its head, drawn at random, and 0 in the others, so an element counts
the seen tokens that chose it: a token left out, taken twice or from a wrong slot
moves a count of at most a few by one.  Sums of ones are exact; one quotient, one
product and the rounding of the output are not."""
import numpy as np
import pytest
import torch

import paper_2407_00066_amd as cts
from oracle import block as ob

from _block_helpers import ROUND, assert_within, to_device
from _gpu_helpers import say
from test_gpu_kv_attention import WEIGHTS, make

pytestmark = pytest.mark.gpu


def _run(c, want, max_kv, window=0):
    """The call with a table that has room for max_kv; want: the plan's (how, runs go from tile to tile, in pieces)."""
    page, kvh = c["cache"][0].shape[2], c["cache"][0].shape[1]
    cols = max(c["table"].shape[1], -(-max_kv // page))
    wide = np.full((c["table"].shape[0], cols), 2 ** 30, np.int32)      # columns past the lengths are not used
    wide[:, :c["table"].shape[1]] = c["table"]
    for b, n in enumerate(c["n_kv"]):
        wide[b, -(-int(n) // page):] = 2 ** 30
    cache, table = to_device(c["cache"]), torch.from_numpy(wide).cuda()
    how, few, pieces = cts.kv_attention_plan(c["q"], cache, table, c["max_q"], max_kv, window)
    rows = np.diff(c["q_start"]) * (c["heads"] // kvh)
    tiles = int((-(-rows // 16) * (rows <= 64)).sum()) * kvh             # those that have rows
    assert (how, how == "runs" and tiles > few, pieces > 1) == want, (how, few, pieces, tiles)
    say("kv_attention %s %s d=%d window=%d tiles=%d pieces=%d" % (how, c["dtype"], c["d"], window, tiles, pieces))
    out = cts.kv_attention(c["q"], cache, table, torch.from_numpy(c["n_kv"]).cuda(),
                           q_start=torch.from_numpy(c["q_start"]).cuda(), max_q=c["max_q"], max_kv=max_kv, window=window)
    torch.cuda.synchronize()
    return out


def _sequences(c):
    """(first row, rows, length, slots) of each sequence."""
    page = c["cache"][0].shape[2]
    for b, L in enumerate(c["n_kv"]):
        t = np.arange(int(L))
        yield int(c["q_start"][b]), int(c["q_start"][b + 1] - c["q_start"][b]), int(L), c["table"][b][t // page].astype(np.int64) * page + t % page


def _attention(c, window):
    """ob.attention's three results, a sequence at a time."""
    d, kvh, heads = c["d"], c["cache"][0].shape[1], c["heads"]
    shape = c["q64"].shape
    out, mag, soft = (np.zeros(shape) for _ in range(3))
    kc, ks, vc, vs = c["cache"]
    page = kc.shape[2]
    for q0, n, L, slots in _sequences(c):
        if n == 0 or L == 0:
            continue
        p, o = slots // page, slots % page
        kv = []
        for by, s in ((kc[p, :, o], ks[p, :, o]), (vc[p, :, o // 4, :, o % 4].reshape(L, kvh, d // 2), vs[p, :, o // 4, :, o % 4])):
            codes = np.stack((by & 15, by >> 4), axis=-1).reshape(L, kvh, d)
            kv.append(ob.dequantize(codes, s))
        pos, t = L - n + np.arange(n), np.arange(L)
        seen = (t <= pos[:, None]) & ((t > pos[:, None] - window) if window else True)
        live = pos >= 0
        for h in range(heads):
            k, v = (a[:, h // (heads // kvh)] for a in kv)
            q = c["q64"][q0:q0 + n, h]
            s = np.where(seen, d ** -0.5 * (q @ k.T), -np.inf)
            e = np.where(seen, (d + 8) * 2.0 ** -24 * d ** -0.5 * (np.abs(q) @ np.abs(k).T), 0).max(1)
            w = np.exp(s - np.where(live, s.max(1), 0)[:, None])
            w /= np.where(live, w.sum(1), 1)[:, None]
            out[q0:q0 + n, h], mag[q0:q0 + n, h] = w @ v, w @ np.abs(v)
            soft[q0:q0 + n, h] = mag[q0:q0 + n, h] * (4 * e + (seen.sum(1) + d) * 2.0 ** -24)[:, None]
    return out, mag, soft


def _check(c, want, max_kv, window=0):
    out = _run(c, want, max_kv, window)
    ref, mag, soft = _attention(c, window)
    assert_within(out, ref, 1.01 * (ROUND[c["dtype"]] * np.abs(ref) + WEIGHTS[c["dtype"]] * mag + soft) + 1e-30, "kv_attention")


def _check_counts(c, want, max_kv, window=0, seed=0):
    kvh, page, d = c["cache"][0].shape[1], c["cache"][0].shape[2], c["d"]
    rng = np.random.default_rng(seed)
    pages = c["cache"][0].shape[0]
    pick = rng.integers(0, d, (pages * page, kvh))                       # the element that a slot's head has a 1 in
    codes = np.zeros((pages * page, kvh, d), np.uint8)
    np.put_along_axis(codes, pick[:, :, None], 2, axis=2)
    by = (codes[:, :, 0::2] | (codes[:, :, 1::2] << 4)).reshape(pages, page // 4, 4, kvh, d // 8, 4)
    c["cache"][2][...] = by.transpose(0, 3, 1, 4, 2, 5)
    c["cache"][3][...] = 127
    c["q"] = torch.zeros_like(c["q"])
    out = _run(c, want, max_kv, window)
    ref = np.zeros(c["q64"].shape)
    group = c["heads"] // kvh
    for q0, n, L, slots in _sequences(c):
        chosen = np.zeros((L + 1, kvh, d))
        np.put_along_axis(chosen[1:], pick[slots][:, :, None], 1, axis=2)
        chosen = chosen.cumsum(0)
        for j in range(n):
            P = L - n + j
            if P >= 0:
                lo = max(0, P - window + 1) if window else 0
                ref[q0 + j] = np.repeat((chosen[P + 1] - chosen[lo]) / (P + 1 - lo), group, axis=0)
    assert_within(out, ref, (1.01 * ROUND[c["dtype"]] + 2.0 ** -22) * ref, "counts")


def _lengths(rng, B, top, few_rows):
    """Sequences of all lengths, and of few and no rows; some empty, and some with many rows that other kernels take."""
    n_kv = rng.integers(1, top, B)
    n_q = np.minimum(rng.integers(1, few_rows + 1, B), n_kv)
    n_kv[0] = top
    if B > 8:
        n_kv[1], n_q[2], n_kv[3], n_q[3] = 0, 0, 33, 33                  # nothing cached; no rows; none but its own
        n_q[1] = 1
        n_kv[5], n_q[5] = 200, 80                                        # many rows
    return n_q.tolist(), n_kv.tolist()


KINDS = [("bf16", 64), ("bf16", 128), ("bf16", 256), ("f32", 64), ("f32", 128), ("f32", 256)]


@pytest.mark.parametrize("dtype,d", KINDS)
@pytest.mark.parametrize("B,kvh,group,few_rows,top,max_kv", [
    (40, 2, 1, 1, 900, 9000), (24, 3, 4, 9, 500, 9000), (13, 7, 2, 3, 1500, 12000), (70, 1, 3, 2, 400, 9000)])
def test_runs_from_tile_to_tile(B, kvh, group, few_rows, top, max_kv, dtype, d):
    n_q, n_kv = _lengths(np.random.default_rng(B + d), B, top, few_rows)
    in_pieces = dtype == "bf16" and max(n_q) * group > 64
    c = make(n_q, n_kv, group * kvh, kvh, d, 16, dtype, seed=B + d)
    pieces = in_pieces and cts.kv_attention_plan(c["q"], to_device(c["cache"]), torch.zeros(B, max_kv // 16), c["max_q"], max_kv)[2] > 1
    _check(c, ("runs", True, pieces), max_kv)
    _check_counts(c, ("runs", True, pieces), max_kv, seed=B)


@pytest.mark.parametrize("dtype,d", KINDS)
@pytest.mark.parametrize("B,kvh,few_rows,window,top", [(20, 4, 1, 3000, 5000), (12, 6, 20, 3500, 4200)])
def test_windows_in_runs_from_tile_to_tile(B, kvh, few_rows, window, top, dtype, d):
    """Windows wide enough for runs, over sequences that are longer."""
    n_q, n_kv = _lengths(np.random.default_rng(B + d), B, top, few_rows)
    n_q[3], n_q[5], n_kv[5] = few_rows, few_rows, top - 1
    c = make(n_q, n_kv, kvh, kvh, d, 32, dtype, seed=B + d)
    want = ("runs", True, False)
    _check(c, want, 20000, window)
    _check_counts(c, want, 20000, window, seed=B)


@pytest.mark.parametrize("window", [0, 1900])
@pytest.mark.parametrize("dtype,d", KINDS)
@pytest.mark.parametrize("n_q,n_kv,kvh,group", [([1], [4099], 1, 1), ([1], [5000], 8, 4), ([3, 1, 2], [2500, 40, 2111], 2, 8),
                                                ([30], [2777], 3, 2), ([1] * 9, [100, 3000, 1, 32, 2049, 700, 2500, 9, 0], 7, 1)])
def test_few_tiles_in_runs_of_their_own(n_q, n_kv, kvh, group, dtype, d, window):
    c = make(n_q, n_kv, group * kvh, kvh, d, 16, dtype, seed=d + kvh)
    if window and len(n_q) > 8:
        window = 2600
    if window and kvh == 8:
        window = 4000
    want = ("runs", False, False)
    _check(c, want, 30000, window)
    _check_counts(c, want, 30000, window, seed=d)


@pytest.mark.parametrize("dtype,d", KINDS)
@pytest.mark.parametrize("B,kvh,group,few_rows", [(64, 8, 1, 1), (33, 8, 4, 1), (128, 4, 2, 1), (128, 3, 3, 4), (40, 5, 12, 2),
                                                  (2, 200, 1, 1), (1, 300, 2, 1), (9, 14, 16, 4)])
def test_whole_tiles_by_length(B, kvh, group, few_rows, dtype, d):
    rng = np.random.default_rng(B + d)
    n_q, n_kv = _lengths(rng, B, 700 if kvh < 100 else 150, few_rows)
    if B > 8:
        n_q[5], n_kv[5] = 1, 650                                         # (no prompts here: tiles are counted by the largest sequence)
        n_q[3] = 1
        n_kv[6:B:3] = [320] * len(n_kv[6:B:3])                           # equal lengths
        n_q = [min(a, b) if b else a for a, b in zip(n_q, n_kv)]
        n_q[4] = min(few_rows, n_kv[4])
        n_q[7], n_kv[7] = few_rows, 400
    want = ("by length", False, False)
    c = make(n_q, n_kv, group * kvh, kvh, d, 16, dtype, seed=B + d)
    _check(c, want, 1100)
    _check_counts(c, want, 1100, seed=B)


@pytest.mark.parametrize("dtype,d", KINDS)
@pytest.mark.parametrize("B,kvh,max_kv", [(5, 3, 800), (150, 2, 3000), (130, 4, 8000)])
def test_whole_tiles_in_the_batchs_order(B, kvh, max_kv, dtype, d):
    n_q, n_kv = _lengths(np.random.default_rng(B), B, 600, 2)
    if B > 8:
        n_q[5] = n_q[3] = 2
    c = make(n_q, n_kv, 2 * kvh, kvh, d, 16, dtype, seed=B)
    _check(c, ("whole", False, False), max_kv)
    _check_counts(c, ("whole", False, False), max_kv, seed=B)


# a step of the prompt kernel is 8192 / d tokens, a tile 128 rows; short sequences leave pieces without steps
@pytest.mark.parametrize("window", [0, 2200])
@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("n_q,n_kv,kvh,group", [([70], [3000], 1, 1), ([128, 65, 3], [3500, 80, 90], 2, 1), ([33, 90], [2222, 95], 2, 4),
                                                ([200], [150], 1, 2), ([129, 77], [129, 4000], 3, 1)])
def test_prompts_in_pieces(n_q, n_kv, kvh, group, d, window):
    c = make(n_q, n_kv, group * kvh, kvh, d, 16, seed=d + kvh)
    page_room = 9000
    how = cts.kv_attention_plan(c["q"], to_device(c["cache"]), torch.zeros(len(n_q), page_room // 16), c["max_q"], page_room, window)[0]
    _check(c, (how, False, True), page_room, window)
    _check_counts(c, (how, False, True), page_room, window, seed=d)


@pytest.mark.parametrize("window", [0, 100])
@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("n_q,n_kv,kvh,group", [([64, 65, 66], [64, 65, 66], 1, 1), ([300, 1, 257], [300, 700, 500], 2, 1),
                                                ([17, 16], [500, 300], 1, 4), ([700], [1500], 9, 2), ([90, 200], [50, 900], 2, 3)])
def test_prompts_count_their_tokens(n_q, n_kv, kvh, group, d, window):
    """The prompt kernel is bf16 only: what its weights' rounding would hide, counts show."""
    c = make(n_q, n_kv, group * kvh, kvh, d, 16, seed=d + kvh)
    plan = cts.kv_attention_plan(c["q"], to_device(c["cache"]), torch.from_numpy(c["table"]), c["max_q"], max(n_kv), window)
    assert plan[2] > 0
    _check_counts(c, (plan[0], False, plan[2] > 1), max(n_kv), window, seed=d)


@pytest.mark.parametrize("window", [0, 2200])
@pytest.mark.parametrize("d", [64, 128, 256])
def test_nan_in_prompts_in_pieces(d, window):
    """NaN keys and values that some rows see and others do not, in pieces of a tile's tokens."""
    n_q, L, max_kv = 100, 2500, 9000
    c = make([n_q], [L], 2, 1, d, 16, seed=d)
    ref, mag, soft = _attention(c, window)
    page = 16
    cut = L - 40
    spoiled = [cut] + ([L - n_q - window + 20] if window else [])
    for i, t in enumerate(spoiled):
        p, o = int(c["table"][0][t // page]), t % page
        c["cache"][3][p, :, o // 4, :, o % 4] = 255
        if i == 0:
            c["cache"][1][p, :, o] = 255
    out = _run(c, (cts.kv_attention_plan(c["q"], to_device(c["cache"]), torch.zeros(1, max_kv // 16), n_q, max_kv, window)[0], False, True),
               max_kv, window)
    pos = L - n_q + np.arange(n_q)
    first = np.maximum(0, pos - window + 1) if window else 0 * pos
    hit = np.array([any(f <= t <= p for t in spoiled) for f, p in zip(first, pos)])
    assert hit.any() and not hit.all()
    got = out.double().cpu().numpy()
    assert np.isnan(got[hit]).all()
    w, m, s = ref[~hit], mag[~hit], soft[~hit]
    assert_within(got[~hit], w, 1.01 * (ROUND["bf16"] * np.abs(w) + WEIGHTS["bf16"] * m + s) + 1e-30, "rows that see no NaN")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n_q,n_kv,max_kv", [([40], [70], 70), ([1], [3000], 30000), ([100], [150], 150)])
def test_nan_blocks_of_wide_heads(n_q, n_kv, max_kv, dtype):
    """One NaN block of a seen value of a head of 256: its 32 elements, and no others."""
    c = make(n_q, n_kv, 2, 2, 256, 16, dtype, seed=n_kv[0])
    t = 20
    p, o = int(c["table"][0][t // 16]), t % 16
    c["cache"][3][p, 1, o // 4, 5, o % 4] = 255
    c["table"] = np.concatenate((c["table"], np.zeros((1, max(0, max_kv // 16 - c["table"].shape[1])), np.int32)), axis=1)
    cache = to_device(c["cache"])
    say("kv_attention NaN block, heads of 256, %s %s" % (n_q, n_kv))
    out = cts.kv_attention(c["q"], cache, torch.from_numpy(c["table"]).cuda(), torch.from_numpy(c["n_kv"]).cuda(),
                           q_start=torch.from_numpy(c["q_start"]).cuda(), max_q=n_q[0], max_kv=max_kv)
    see = torch.arange(n_kv[0] - n_q[0], n_kv[0], device="cuda") >= t
    want = torch.zeros_like(out, dtype=torch.bool)
    want[see, 1, 160:192] = True
    assert torch.equal(torch.isnan(out), want)


@pytest.mark.parametrize("n_q,dtype", [(70, "bf16"), (70, "f32"), (20, "bf16")])
def test_pages_past_32_bits(n_q, dtype):
    """Prompts whose pages' bytes lie past 2^32, beside one at the cache's start."""
    pages, page, kvh, d = 2200, 1024, 32, 128                            # 4.6 GB of key codes
    cache = cts.kv_cache(pages, page, kvh, d)
    rng = np.random.default_rng(n_q)
    slots = np.concatenate(((pages - 1) * page + np.arange(n_q), np.arange(n_q)))
    k, v = (torch.from_numpy(rng.standard_normal((2 * n_q, kvh, d)).astype(np.float32)).cuda() for _ in range(2))
    cts.kv_write(cache, k, v, torch.from_numpy(slots).cuda())
    small = [torch.zeros_like(t[:2]) for t in (cache.k_codes, cache.k_scales, cache.v_codes, cache.v_scales)]
    for t, s in zip((cache.k_codes, cache.k_scales, cache.v_codes, cache.v_scales), small):
        s[0], s[1] = t[pages - 1], t[0]
    q = torch.from_numpy(rng.standard_normal((2 * n_q, kvh, d)).astype(np.float32)).to(dtype=torch.float32 if dtype == "f32" else torch.bfloat16).cuda()
    n_kv = torch.tensor([n_q, n_q], dtype=torch.int32, device="cuda")
    start = torch.tensor([0, n_q, 2 * n_q], dtype=torch.int32, device="cuda")
    say("kv_attention past 32 bits %s n=%d" % (dtype, n_q))
    tables = [torch.tensor(t, dtype=torch.int32, device="cuda") for t in ([[pages - 1], [0]], [[0], [1]])]
    got = cts.kv_attention(q, cache, tables[0], n_kv, q_start=start, max_q=n_q)
    want = cts.kv_attention(q, cts.KVCache(*small), tables[1], n_kv, q_start=start, max_q=n_q)
    assert torch.equal(got, want) and bool(want.any())
