"""The decoder-block oracle against values worked out by hand, closed forms and
planted mistakes (CPU)."""
import numpy as np
import pytest

from oracle import block as ob


def test_quantize_worked_example():
    # largest 6: scale 2^0 (byte 127); every magnitude and its ties
    x = np.zeros(32)
    x[:16] = [0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.0, -0.25, -0.75, -0.2501, 0.2501, -5.01, 0.49, 0.0, -0.0]
    c, s = ob.quantize(x)
    assert s.tolist() == [127]
    assert c[:16].tolist() == [0, 2, 2, 4, 4, 6, 6, 7, 8, 10, 9, 1, 15, 1, 0, 8]


@pytest.mark.parametrize("top,byte,code", [(6.99, 127, 7), (7.0, 128, 6), (8.0, 128, 6), (4.0, 127, 6), (3.5, 127, 6),
                                           (3.49, 126, 7), (1.0, 125, 6), (0.0, 1, 0), (2.0 ** -140, 1, 0),
                                           (2.0 ** -126, 1, 2), (3.3e38, 252, 7), (2.0 ** 127, 252, 6)])
def test_quantize_scale(top, byte, code):
    x = np.zeros(32)
    x[5] = top
    c, s = ob.quantize(x)
    assert s[0] == byte and c[5] == code


@pytest.mark.parametrize("bad", [np.nan, np.inf, -np.inf])
def test_quantize_not_finite(bad):
    x = np.ones(64)
    x[40] = bad
    c, s = ob.quantize(x)
    assert s[1] == 255 and s[0] != 255
    v = ob.dequantize(c, s)
    assert np.isnan(v[32:]).all() and not np.isnan(v[:32]).any()


def test_round_trip_error():
    # an element is off by at most half its step: a sixth of itself, or a quarter of the unit
    rng = np.random.default_rng(0)
    x = rng.standard_normal((50, 128)) * np.exp(rng.standard_normal((50, 1)) * 5)
    c, s = ob.quantize(x)
    v = ob.dequantize(c, s)
    unit = np.repeat(np.exp2(s.astype(float) - 127), 32, axis=-1)
    assert (np.abs(v - x) <= np.maximum(np.abs(x) / 5, unit / 4) + 1e-12).all()
    c2, s2 = ob.quantize(v)                           # what was read back is stored as it is
    assert np.array_equal(ob.dequantize(c2, s2), v)


def test_write_read():
    rng = np.random.default_rng(1)
    cache = ob.empty_cache(3, 16, 2, 64)
    k, v = rng.standard_normal((2, 5, 2, 64))
    slots = [47, 0, -1, 17, 48]
    ob.write(cache, k, v, slots)
    rk, rv = ob.read(cache, slots)
    for t in (0, 1, 3):
        assert np.array_equal(rk[t], ob.dequantize(*ob.quantize(k[t])))
        assert np.array_equal(rv[t], ob.dequantize(*ob.quantize(v[t])))
    assert not rk[[2, 4]].any() and not rv[[2, 4]].any()
    others = [s for s in range(48) if s not in slots]
    assert not ob.read(cache, others)[0].any()


def _attend(n_kv, q_start, window=0, seed=2, heads=4, plant=None):
    rng = np.random.default_rng(seed)
    cache = ob.empty_cache(8, 16, 2, 64)
    k, v = rng.standard_normal((2, 128, 2, 64))
    ob.write(cache, k, v, range(128))
    table = np.array([[7, 2, 5], [0, 1, 3]])
    q = rng.standard_normal((q_start[-1], heads, 64))
    return q, cache, table, ob.attention(q, cache, table, n_kv, q_start, 0.125, window)[0]


def test_attention_one_token_is_its_value():
    q, cache, table, out = _attend([1, 1], [0, 1, 2])
    for b in range(2):
        _, v = ob.read(cache, [table[b][0] * 16])
        assert np.allclose(out[b], np.repeat(v[0], 2, axis=0))


def test_attention_matches_dense_softmax():
    q, cache, table, out = _attend([37, 48], [0, 3, 8], window=9)
    for b, (L, q0, q1) in enumerate(((37, 0, 3), (48, 3, 8))):
        K, V = ob.read(cache, [table[b][t // 16] * 16 + t % 16 for t in range(L)])
        s = np.einsum("qhd,thd->hqt", q[q0:q1], np.repeat(K, 2, axis=1)) * 0.125
        pos = L - (q1 - q0) + np.arange(q1 - q0)
        t = np.arange(L)
        hide = (t[None] > pos[:, None]) | (t[None] <= pos[:, None] - 9)
        s[:, hide] = -np.inf
        w = np.exp(s - s.max(-1, keepdims=True))
        w /= w.sum(-1, keepdims=True)
        assert np.allclose(out[q0:q1], np.einsum("hqt,thd->qhd", w, np.repeat(V, 2, axis=1)))


def test_attention_empty_rows():
    _, _, _, out = _attend([0, 2], [0, 2, 6])         # nothing cached; four queries over two tokens
    assert not out[:4].any() and out[4:].any()


def test_block_norm_closed_form():
    x, y = np.full((1, 4), 3.0), np.array([[2.0, -2.0, 2.0, -2.0]])
    h, n, _ = ob.block_norm(x, np.ones(4), y, post=np.full(4, 5.0), gate=np.array([1.0, 0, 1, 0]), scale=0.2, eps=0.0)
    assert np.allclose(h, [[4, 3, 4, 3]]) and np.allclose(n, h / np.sqrt(12.5))


def test_rotary_quarter_turn_and_norm():
    cos, sin = np.zeros((2, 8)), np.ones((2, 8))
    x = np.arange(16.0).reshape(1, 1, 16)
    out, _ = ob.rotary(x, cos, sin, [[0]], [8])
    assert np.array_equal(out[0, 0], np.concatenate((-x[0, 0, 8:], x[0, 0, :8])))
    out, _ = ob.rotary(x, cos, sin, [[0]], [8], interleaved=True)
    assert out[0, 0, :4].tolist() == [-1, 0, -3, 2]
    rng = np.random.default_rng(3)
    ang = rng.standard_normal((5, 16))
    x = rng.standard_normal((4, 3, 32))
    out, _ = ob.rotary(x, np.cos(ang), np.sin(ang), rng.integers(0, 5, (3, 4)), [4, 5, 7])
    assert np.allclose((out ** 2).sum(-1), (x ** 2).sum(-1))


@pytest.mark.parametrize("mistake", ["scale", "mask", "head", "axis"])
def test_planted_mistakes_are_seen(mistake, monkeypatch):
    """A wrong oracle differs from the right one by more than any tolerance used."""
    q, cache, table, right = _attend([37, 48], [0, 3, 8])
    if mistake == "scale":
        wrong = ob.attention(q, cache, table, [37, 48], [0, 3, 8], 0.13)[0]
    elif mistake == "mask":
        wrong = ob.attention(q, cache, table, [36, 47], [0, 3, 8], 0.125)[0]
    elif mistake == "head":
        wrong = ob.attention(q[:, ::-1], cache, table, [37, 48], [0, 3, 8], 0.125)[0]
    else:
        rng = np.random.default_rng(4)
        ang, x, pos = rng.standard_normal((9, 16)), rng.standard_normal((4, 3, 32)), rng.integers(0, 9, (2, 4))
        right = ob.rotary(x, np.cos(ang), np.sin(ang), pos, [8, 8])[0]
        wrong = ob.rotary(x, np.cos(ang), np.sin(ang), pos, [9, 7])[0]
    assert np.abs(wrong - right).max() > 0.05
