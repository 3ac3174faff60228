"""cts_kv_tree_attention on tiles of 32 and 64 rows under every way its work is dealt out: whole with eight and
with four waves, by work, and cut, with and without a window.  Such tiles are for batches of more work than a
test needs, so wide tables make loose bounds; sequences have every number of drafts, so that tiles of one to four
groups of 16 rows stand side by side."""
import numpy as np
import pytest
import torch

from _draft_helpers import call, check, make
from _gpu_helpers import say
from test_gpu_tree_attention import _poison
from test_gpu_tree_schedules import _plan, _widen

pytestmark = pytest.mark.gpu


def _uneven(B, most, top, long, seed):
    """Drafts and tokens before them: 0 to `most` drafts, every number of them among the first; `long` sequences
    far longer than `top`."""
    rng = np.random.default_rng(seed)
    n_q, n_past = rng.integers(0, most + 1, B), rng.integers(0, top, B)
    first = np.arange(most, 0, -1)[:B]
    n_q[:len(first)] = first
    n_past[::9] = 0
    for b, n in long:
        n_past[b] = n
    return n_q.tolist(), n_past.tolist()


def _batch(B, kvh, heads, d, dtype, most, cols, top, long=(), wild=False):
    n_q, n_past = _uneven(B, most, top, long, B + d + most)
    return _widen(make(n_q, n_past, heads, kvh, d, 16, dtype, seed=B + d, wild=wild), cols)


# more tiles than compute units: those with most work first
@pytest.mark.parametrize("B,kvh,heads,d,dtype,most,cols,rows,waves", [
    (64, 8, 32, 128, "bf16", 16, 40, 64, 4), (64, 8, 32, 64, "bf16", 16, 40, 64, 4), (200, 8, 32, 128, "bf16", 8, 20, 32, 4),
    (200, 8, 32, 64, "bf16", 8, 20, 32, 4), (200, 8, 16, 256, "bf16", 16, 30, 32, 8), (200, 4, 16, 64, "f32", 8, 30, 32, 4),
    (200, 4, 16, 128, "f32", 8, 30, 32, 4)])
def test_by_work(B, kvh, heads, d, dtype, most, cols, rows, waves):
    c = _batch(B, kvh, heads, d, dtype, most, cols, 150)
    assert _plan(c) == (rows, "by work", waves)
    check(c)


# more sequences than are ordered; few tiles, whose workgroups have eight waves
@pytest.mark.parametrize("B,kvh,heads,d,dtype,most,cols,rows,waves", [
    (300, 2, 8, 128, "bf16", 16, 32, 64, 4), (300, 2, 8, 64, "bf16", 16, 32, 64, 4), (300, 2, 8, 128, "bf16", 8, 64, 32, 4),
    (60, 4, 16, 128, "bf16", 16, 80, 64, 8), (60, 4, 16, 64, "bf16", 16, 80, 64, 8), (30, 8, 32, 128, "bf16", 8, 80, 32, 8),
    (60, 4, 16, 128, "f32", 8, 80, 32, 8)])
def test_whole(B, kvh, heads, d, dtype, most, cols, rows, waves):
    c = _batch(B, kvh, heads, d, dtype, most, cols, 200, [(2, 490), (7, 470)], wild=B == 60)
    assert _plan(c) == (rows, "whole", waves)
    check(c)


# more than 64 tiles, with fewer that have work than run at a time and with more
@pytest.mark.parametrize("B,kvh,heads,d,dtype,most,cols,rows,waves", [
    (80, 2, 8, 128, "bf16", 16, 300, 64, 4), (80, 2, 8, 64, "bf16", 16, 300, 64, 4), (70, 6, 24, 128, "bf16", 16, 300, 64, 4),
    (70, 6, 24, 64, "bf16", 8, 300, 32, 4), (80, 2, 8, 128, "f32", 8, 600, 32, 4), (80, 2, 4, 256, "bf16", 16, 300, 32, 8)])
def test_many_tiles_cut(B, kvh, heads, d, dtype, most, cols, rows, waves):
    c = _batch(B, kvh, heads, d, dtype, most, cols, 250, [(3, 4000), (B - 3, 1500), (5, 999)])
    assert _plan(c) == (rows, "cut", waves)
    check(c)


# a row's position says where its window begins: rows of a tile begin at different tokens
@pytest.mark.parametrize("B,kvh,heads,d,dtype,most,cols,window,how,rows", [
    (250, 8, 16, 128, "bf16", 32, 60, 70, "by work", 64), (250, 8, 16, 64, "bf16", 32, 60, 70, "by work", 64),
    (200, 8, 32, 128, "f32", 8, 40, 150, "by work", 32), (250, 8, 16, 256, "bf16", 16, 60, 120, "by work", 32),
    (60, 4, 16, 128, "bf16", 16, 200, 1300, "whole", 64)])
def test_windows(B, kvh, heads, d, dtype, most, cols, window, how, rows):
    n_q, n_past = _uneven(B, most, 300, [(1, 2 * window), (3, 2 * window + 13), (4, window + 3)], B + d)
    if most == 32:
        n_q = [n if b < 33 else n % 4 for b, n in enumerate(n_q)]
    c = _widen(make(n_q, n_past, heads, kvh, d, 16, dtype, seed=d), cols)
    assert _plan(c, window)[:2] == (rows, how)
    check(c, window)


@pytest.mark.parametrize("d,most,rows", [(128, 16, 64), (64, 16, 64), (128, 8, 32)])
def test_windows_of_cut_tiles(d, most, rows):
    n_q, n_past = _uneven(32, most, 120, [(0, 4100), (1, 2098), (4, 2300), (6, 3001)], d + most)
    c = _widen(make(n_q, n_past, 16, 4, d, 16, seed=d + most), 400)
    assert _plan(c, 2100) == (rows, "cut", 4)
    check(c, 2100)


@pytest.mark.parametrize("B,kvh,heads,d,most,cols,how", [(64, 8, 32, 128, 16, 40, "by work"), (300, 2, 8, 64, 16, 32, "whole"),
                                                         (60, 4, 16, 128, 16, 80, "whole")])
def test_whole_tiles_keep_their_bits_beside_others(B, kvh, heads, d, most, cols, how):
    """A sequence among others under one plan: with other neighbours, and with none that have drafts, its rows have the same bits."""
    c = _batch(B, kvh, heads, d, "bf16", most, cols, 200)
    assert _plan(c)[:2] == (64, how)
    a = call(c)
    other = dict(c, n_kv=c["n_kv"].copy())
    kept = [0, 3, 5, B - 1]
    for b in range(B):
        if b not in kept:
            other["n_kv"][b] = c["n_kv"][B - 1 - b] if b % 2 else 0
    room = (c["table"] != 2 ** 30).sum(1) * 16                   # (tokens that a sequence's own pages hold)
    other["n_kv"] = np.minimum(other["n_kv"], room).astype(np.int32)
    other["n_kv"][kept] = c["n_kv"][kept]
    b_out = call(other)
    rows = [r for b in kept for r in range(c["q_start"][b], c["q_start"][b + 1])]
    assert rows and torch.equal(a[rows], b_out[rows]) and not torch.equal(a, b_out)
    # alone: the other sequences have no rows
    b = 3
    lo, hi = int(c["q_start"][b]), int(c["q_start"][b + 1])
    start = np.where(np.arange(B + 1) <= b, lo, hi).astype(np.int32)
    out = torch.full_like(a, 5.0)
    call(dict(c, q_start=start), out=out)
    assert hi > lo and torch.equal(out[lo:hi], a[lo:hi])
    assert bool((out[:lo] == 5).all()) and bool((out[hi:] == 5).all())


# (64 rows of one key/value head: 16 drafts of 4 heads, or 32 of 2)
@pytest.mark.parametrize("B,kvh,heads,d,dtype,most,cols,window,how,rows", [
    (60, 4, 16, 128, "bf16", 16, 80, 0, "whole", 64), (60, 4, 16, 64, "bf16", 16, 80, 0, "whole", 64),
    (64, 8, 32, 64, "bf16", 16, 40, 0, "by work", 64), (80, 2, 8, 128, "bf16", 16, 300, 0, "cut", 64),
    (80, 2, 8, 64, "bf16", 16, 300, 0, "cut", 64), (80, 2, 4, 256, "bf16", 16, 300, 0, "cut", 32),
    (60, 4, 16, 128, "f32", 8, 80, 0, "whole", 32), (250, 8, 16, 64, "bf16", 32, 60, 70, "by work", 64),
    (32, 4, 16, 128, "bf16", 16, 400, 2100, "cut", 64)])
def test_nan_in_hidden_places(B, kvh, heads, d, dtype, most, cols, window, how, rows):
    """NaN drafts, NaN tokens before a window and NaN past the ends: rows that do not see one come out bit for bit as
    without them, the others as NaN."""
    n_q, n_past = _uneven(B, most, 100, [(1, window + 60), (3, window + 200)], B + d)
    if most == 32:
        n_q = [n if b < 33 else n % 4 for b, n in enumerate(n_q)]
    c = _widen(make(n_q, n_past, heads, kvh, d, 16, dtype, seed=d), cols)
    assert _plan(c, window)[:2] == (rows, how)
    clean = call(c, window)
    sees = np.zeros(len(c["mask"]), bool)
    for b, (n, past) in enumerate(zip(n_q, n_past)):
        sick = [i for i in range(n) if (i + b) % 5 == 2]
        early = 30 if window and past > window else -1           # a token that only rows near the first draft may see
        _poison(c, b, [past + i for i in sick] + [early] * (early >= 0), "kv")
        last = int(c["table"][b][(past + n - 1) // 16]) if past + n else -1
        for o in range((past + n - 1) % 16 + 1, 16 if last >= 0 else 0):
            c["cache"][1][last, :, o], c["cache"][3][last, :, o // 4, :, o % 4] = 255, 255
        for r in range(c["q_start"][b], c["q_start"][b + 1]):
            sees[r] = any(int(c["mask"][r][i // 32]) >> (i % 32) & 1 for i in sick) or \
                (early >= 0 and early > max(int(c["pos"][r]), past) - window)
    say("kv_tree_attention over NaN, %s tiles of %d rows, d=%d %s window=%d" % (how, rows, d, dtype, window))
    out = call(c, window)
    hit = torch.isnan(out).flatten(1)
    assert sees.any() and not sees.all() and np.array_equal(hit.all(1).cpu().numpy(), sees)
    well = torch.from_numpy(~sees).cuda()
    assert not hit[well].any() and torch.equal(out[well], clean[well])


@pytest.mark.parametrize("B,kvh,heads,most,cols,how", [(60, 4, 16, 16, 80, "whole"), (80, 2, 8, 16, 300, "cut")])
def test_pages_outside_the_cache(B, kvh, heads, most, cols, how):
    c = _batch(B, kvh, heads, 128, "bf16", most, cols, 200)
    assert _plan(c)[:2] == (64, how)
    clean = call(c)
    sick = [b for b in range(1, B, 7) if c["n_kv"][b] > np.diff(c["q_start"])[b]]
    for b in sick:
        c["table"][b, 0] = (-1, 2 ** 31 - 1, len(c["cache"][0]))[b % 3]
    out = call(c)
    for b in range(B):
        at = slice(int(c["q_start"][b]), int(c["q_start"][b + 1]))
        assert torch.isnan(out[at]).all() if b in sick else torch.equal(out[at], clean[at]), b


@pytest.mark.parametrize("B,kvh,heads,d,dtype,most,cols,how", [
    (60, 4, 16, 128, "bf16", 16, 80, "whole"), (80, 2, 8, 64, "bf16", 16, 300, "cut"), (60, 4, 16, 128, "f32", 8, 80, "whole"),
    (5, 2, 8, 128, "bf16", 16, 40, "whole")])
def test_queries_that_are_no_numbers(B, kvh, heads, d, dtype, most, cols, how):
    """A NaN or an infinity in a query makes that query's head NaN (zeros, where every score is -inf) and no bit of another
    row different."""
    c = _batch(B, kvh, heads, d, dtype, most, cols, 200)
    assert _plan(c)[1] == how
    clean = call(c)
    q = c["q"].clone()
    sick = [(r, r % heads) for r in range(1, len(q), 3)]
    for i, (r, h) in enumerate(sick):
        q[r, h, (7 * r) % d] = (float("nan"), float("inf"), float("-inf"))[i % 3]
    say("kv_tree_attention of NaN queries, %s" % how)
    out = call(c, q=q)
    well = torch.ones(q.shape[:2], dtype=torch.bool, device="cuda")
    for i, (r, h) in enumerate(sick):
        well[r, h] = False
        assert torch.isnan(out[r, h]).all() or i % 3 and not out[r, h].any()
    assert torch.equal(out[well], clean[well])


@pytest.mark.parametrize("most,cols,how", [(16, 80, "whole"), (16, 300, "cut")])
def test_lengths_and_rows_outside_their_bounds(most, cols, how):
    """A kv_len past max_kv counts as that, one below 0 as 0; rows are clamped to those that there are, and a sequence whose
    end lies before its start has none."""
    B, kvh, heads, d = (60, 4, 16, 128) if how == "whole" else (80, 2, 8, 64)
    c = _batch(B, kvh, heads, d, "bf16", most, cols, 200)
    assert _plan(c)[:2] == (64, how)
    room, T = cols * 16, len(c["q"])
    over = dict(c, n_kv=c["n_kv"].copy(), q_start=c["q_start"].copy())
    over["n_kv"][[0, 7, 20]] = [-1, -2 ** 31, -5]
    c["n_kv"][[0, 7, 20]] = 0
    # a last sequence of all the table's tokens (pages that others hold too)
    c["table"][B - 1], c["n_kv"][B - 1], over["n_kv"][B - 1] = np.arange(cols) % len(c["cache"][0]), room, 2 ** 31 - 1
    over["table"] = c["table"]
    over["q_start"][0], over["q_start"][-1] = -77, 2 ** 31 - 1
    assert c["q_start"][0] == 0 and c["q_start"][-1] == T
    say("kv_tree_attention of lengths past their bounds, %s" % how)
    assert torch.equal(call(over), call(c))
    check(c)
    # sequence 3 has no rows, sequence 4 from where it begins, more than max_q: those past it stay as they were
    back = dict(c, q_start=c["q_start"].copy())
    back["q_start"][4] = back["q_start"][3] - 5
    a = torch.full_like(c["q"], 5.0)
    call(back, out=a)
    lo, hi = int(back["q_start"][4]), int(back["q_start"][5])
    assert hi - lo > most and bool((a[lo + most:hi] == 5).all()) and not bool((a[lo:lo + most] == 5).all(2).any())
    same = torch.equal(a[hi:], call(c)[hi:])                     # (cut, the lengths of pieces follow from all work)
    assert same or how == "cut"
