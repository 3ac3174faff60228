"""The oracle of the drafted-token operators against closed forms and the oracles beside it."""
import numpy as np
import pytest

from oracle import block as ob


def _cache(rng, pages, page, heads, d):
    c = ob.empty_cache(pages, page, heads, d)
    for a in (c[0], c[2]):
        a[...] = rng.integers(0, 256, a.shape)
    for a in (c[1], c[3]):
        a[...] = rng.integers(122, 128, a.shape)
    return c


def _chain(n, words):
    """Masks of drafts that follow each other."""
    m = np.zeros((n, words), np.uint32)
    for j in range(n):
        for i in range(j + 1):
            m[j, i // 32] |= np.uint32(1) << np.uint32(i % 32)
    return m


@pytest.mark.parametrize("window", [0, 9])
def test_a_chain_is_causal_attention(window):
    rng = np.random.default_rng(0)
    cache = _cache(rng, 6, 16, 2, 64)
    n_q, n_kv = [40, 1, 3], [50, 20, 3]
    start = np.concatenate(([0], np.cumsum(n_q)))
    table = np.array([[0, 2, 4, 5], [1, 3, 0, 0], [3, 0, 0, 0]])
    q = rng.standard_normal((44, 4, 64))
    pos = np.concatenate([np.arange(L - n, L) for n, L in zip(n_q, n_kv)])
    mask = np.concatenate([_chain(n, 2) for n in n_q])
    if window:                                                      # of the drafts, the mask alone says
        for b in range(3):
            for j in range(n_q[b]):
                for i in range(max(0, j - window + 1)):
                    mask[start[b] + j, i // 32] &= ~(np.uint32(1) << np.uint32(i % 32))
    got = ob.tree_attention(q, cache, table, n_kv, start, mask, 0.125, window, pos)
    want = ob.attention(q, cache, table, n_kv, start, 0.125, window)
    assert all(np.allclose(a, b, rtol=1e-13, atol=1e-13) for a, b in zip(got, want))


def test_counts_what_a_row_sees():
    """Queries of zero weigh all tokens alike: of tokens worth 1 and 0 the output is the seen share of ones."""
    cache = ob.empty_cache(2, 16, 1, 64)
    ones = [3, 18, 19, 21]
    ob.write(cache, np.zeros((4, 1, 64)), np.ones((4, 1, 64)), ones)
    # 22 tokens, the last 5 (17 .. 21) drafts: 0 <- 1 <- 4, 2 <- 3
    mask = np.array([[1], [0b11], [0b100], [0b1100], [0b10011]], np.uint32)
    out, _, _ = ob.tree_attention(np.zeros((5, 1, 64)), cache, [[0, 1]], [22], [0, 5], mask, 1.0)
    assert np.allclose(out[:, 0, 0], [1 / 18, 2 / 19, 2 / 18, 2 / 19, 3 / 20])
    out, _, _ = ob.tree_attention(np.zeros((5, 1, 64)), cache, [[0, 1]], [22], [0, 5], mask, 1.0, 15, [17, 18, 17, 18, 19])
    assert np.allclose(out[:, 0, 0], [1 / 15, 1 / 15, 2 / 15, 1 / 15, 2 / 15])
    out, _, _ = ob.tree_attention(np.zeros((5, 1, 64)), cache, [[0, 1]], [5], [0, 5], 0 * mask, 1.0)
    assert not out.any()


def test_keep_moves_what_was_there():
    rng = np.random.default_rng(1)
    cache = _cache(rng, 4, 16, 2, 64)
    table = np.array([[2, 0], [1, 3]])
    before = ob.read(cache, np.arange(64))
    # drafts 12 .. 19 of the first, 30 and 31 of the second: 1, 4, 6 kept, the second one
    ob.keep(cache, table, [20, 32], [0, 8, 10], np.array([[1, 4, 6, 3], [1, -1, 0, 0]]), [3, 1])
    after = ob.read(cache, np.arange(64))
    moved = {32 + 12: 32 + 13, 32 + 13: 0, 32 + 14: 2, 48 + 14: 48 + 15}
    for slot in range(64):
        src = moved.get(slot, slot)
        assert all(np.array_equal(a[slot], b[src]) for a, b in zip(after, before)), slot


def test_keep_repeats_and_skips():
    rng = np.random.default_rng(2)
    cache = _cache(rng, 1, 16, 1, 64)
    before = ob.read(cache, np.arange(16))
    ob.keep(cache, np.array([[0]]), [10], [0, 4], np.array([[3, 0, 9, -1, 2]]), [7])
    after = ob.read(cache, np.arange(16))
    for slot in range(16):
        src = {6: 9, 7: 6}.get(slot, slot)
        assert np.array_equal(after[0][slot], before[0][src]) and np.array_equal(after[1][slot], before[1][src])
