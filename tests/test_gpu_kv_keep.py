"""cts_kv_keep against the oracle, byte for byte."""
import numpy as np
import pytest
import torch

import paper_2407_00066_amd as cts
from oracle import block as ob

from _block_helpers import to_device, to_host
from _draft_helpers import drafted, filled, i32
from _gpu_helpers import say

pytestmark = pytest.mark.gpu


def _tables(rng, n_kv, page, spare=2):
    need = [-(-n // page) for n in n_kv]
    order = rng.permutation(sum(need) + spare)
    table, used = np.zeros((len(n_kv), max(need + [1])), np.int32), 0
    for b, n in enumerate(need):
        table[b, :n] = order[used:used + n]
        used += n
    return table, sum(need) + spare


def _check(c, table, n_kv, start, path, n_path):
    want = tuple(a.copy() for a in c)
    dev = to_device(c)
    say("kv_keep kv=%s start=%s path=%s" % (list(n_kv)[:6], list(start)[:6], path.shape))
    cts.kv_keep(dev, i32(table), i32(np.asarray(n_kv, np.int32)), i32(np.asarray(start, np.int32)), i32(path), i32(n_path))
    torch.cuda.synchronize()
    ob.keep(want, table, n_kv, start, path, n_path)
    assert all(np.array_equal(a, b) for a, b in zip(to_host(dev), want))
    return want


@pytest.mark.parametrize("d,kvh,page", [(64, 2, 16), (128, 3, 16), (256, 1, 64), (128, 8, 1024)])
def test_accepted_branches(d, kvh, page):
    rng = np.random.default_rng(d + kvh)
    n_q = [1, 2, 7, 16, 33, 64, 5, 9]
    n_kv = [n + p for n, p in zip(n_q, [0, 1, 15, 16, 31, 200, 14, 0])]
    table, pages = _tables(rng, n_kv, page)
    paths = []
    for n in n_q:
        parents, _ = drafted(rng, n)
        at, path = n - 1, []
        while at >= 0:
            path.insert(0, at)
            at = parents[at]
        paths.append(path)
    most = max(map(len, paths)) + 3
    path = np.array([p + [-1] * (most - len(p)) for p in paths], np.int32)
    n_path = np.array([len(p) for p in paths], np.int32)
    n_path[-2] = 0
    _check(filled(rng, pages, page, kvh, d), table, n_kv, np.concatenate(([0], np.cumsum(n_q))), path, n_path)


@pytest.mark.parametrize("seed", range(4))
def test_any_path(seed):
    """Paths in no order, with repetitions and entries that are no drafts; counts past the row and below 0; drafts that
    begin before the first token; pages outside the cache."""
    rng = np.random.default_rng(seed)
    n_q = rng.integers(0, 40, 6)
    n_kv = rng.integers(0, 60, 6)
    table, pages = _tables(rng, n_kv, 16)
    if seed % 2:
        table[2, -1], table[3, 0], table[4, 0] = -1, 2 ** 30, pages
    path = rng.integers(-3, 45, (6, 50)).astype(np.int32)
    path[0, ::3] = [2 ** 31 - 1, -2 ** 31] * 8 + [0]
    _check(filled(rng, pages, 16, 2, 64), table, n_kv, np.concatenate(([0], np.cumsum(n_q))), path,
           np.array([50, 2 ** 31 - 1, -5, 17, 1, 33], np.int32))


def test_longest_path_and_a_lengths_past_the_table():
    rng = np.random.default_rng(9)
    table, pages = _tables(rng, [700], 16)
    path = rng.permutation(600)[None, :512].astype(np.int32)
    c = filled(rng, pages, 16, 1, 256)
    _check(c, table, [700], [0, 600], path, np.array([512], np.int32))
    # (the table has room for 704)
    a, b = to_device(c), to_device(c)
    cts.kv_keep(a, i32(table), i32(np.array([2 ** 31 - 1], np.int32)), i32(np.array([0, 600], np.int32)), i32(path), i32(np.array([512], np.int32)))
    cts.kv_keep(b, i32(table), i32(np.array([704], np.int32)), i32(np.array([0, 600], np.int32)), i32(path), i32(np.array([512], np.int32)))
    assert all(np.array_equal(x, y) for x, y in zip(to_host(a), to_host(b)))


def test_nothing_to_keep():
    rng = np.random.default_rng(10)
    c = filled(rng, 2, 16, 1, 64)
    _check(c, np.array([[0, 1]], np.int32), [20], [0, 4], np.zeros((1, 0), np.int32), np.array([1], np.int32))
    _check(c, np.zeros((0, 2), np.int32), [], [0], np.zeros((0, 3), np.int32), np.zeros(0, np.int32))
    _check(c, np.array([[0, 1]], np.int32), [20], [7, 3], np.zeros((1, 3), np.int32), np.array([3], np.int32))


def test_past_32_bits():
    n, page = 40000, 1024
    cache = cts.kv_cache(n, page, 2, 256)
    table = torch.tensor([[39999, 17000]], dtype=torch.int32, device="cuda")
    k = torch.randn(4, 2, 256, device="cuda").bfloat16()
    at = torch.tensor([39999 * page + 1022, 39999 * page + 1023, 17000 * page, 17000 * page + 1], device="cuda")
    cts.kv_write(cache, k, -k, at)
    was = cts.kv_read(cache, at)
    say("kv_keep past 32 bits")
    cts.kv_keep(cache, table, i32(np.array([1026], np.int32)), i32(np.array([0, 4], np.int32)), i32(np.array([[1, 3]], np.int32)),
                i32(np.array([2], np.int32)))
    now = cts.kv_read(cache, at)
    for a, b in zip(now, was):
        assert torch.equal(a, b[[1, 3, 2, 3]])


def test_refusals():
    cache = cts.kv_cache(2, 16, 1, 64)
    t = lambda *v: torch.tensor(v, dtype=torch.int32, device="cuda")
    good = [t([0, 1]), t(20), t(0, 4), t([1, 2]), t(2)]
    cts.kv_keep(cache, *good)
    for i, bad, error in [(0, good[0][0], ValueError), (0, good[0].long(), TypeError), (1, t(20, 3), ValueError), (2, t(0, 4, 5), ValueError),
                          (3, t(1, 2), ValueError), (3, t([1, 2], [3, 4]), ValueError), (4, t(2, 2), ValueError),
                          (3, torch.zeros(1, 513, dtype=torch.int32, device="cuda"), cts.CtsError)]:
        args = list(good)
        args[i] = bad
        with pytest.raises(error):
            cts.kv_keep(cache, *args)


def test_unsorted_counts_and_padded_batches():
    """Sequences without drafts, with counts that fall, and lengths below their drafts: what is no draft's place stays."""
    cache = cts.kv_cache(6, 16, 2, 64)
    for a in (cache.k_codes, cache.v_codes, cache.k_scales, cache.v_scales):
        a.random_(0, 250)
    before = [a.copy() for a in to_host(cache)]
    t = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")
    say("kv_keep of padded batches")
    # no drafts; starts that fall back; 3 tokens cached of 5 drafts: draft 4 (token 2) to draft 1's place (before the first token)
    cts.kv_keep(cache, t([[0, 1], [2, 3], [4, 5]]), t([20, 20, 3]), t([4, 4, 0, 5]), t([[0, 1], [1, 0], [2, 4]]), t([2, 2, 2]))
    torch.cuda.synchronize()
    assert all(np.array_equal(a, b) for a, b in zip(to_host(cache), before))
