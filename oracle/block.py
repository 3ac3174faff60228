"""The decoder block's operators (include/cts_block.h) in fp64 numpy, written
from their formulas: the 4-bit cache, the attention over it, block norms and
rotary positions.  Test infrastructure only; shares no code with the library.

Cache arrays are uint8 numpy arrays in the header's layouts, passed as the
tuple (k_codes, k_scales, v_codes, v_scales).
"""
from __future__ import annotations

import numpy as np

MAGNITUDES = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


# ---------------------------------------------------------------- 4-bit blocks
def quantize(x):
    """(codes, scales) of x [..., d]: a code an element, a scale byte a block of 32."""
    x = np.asarray(x, dtype=np.float64)
    blk = x.reshape(x.shape[:-1] + (x.shape[-1] // 32, 32))
    codes = np.zeros(blk.shape, dtype=np.uint8)
    scales = np.zeros(blk.shape[:-1], dtype=np.uint8)
    for at in np.ndindex(*scales.shape):
        b = blk[at]
        if not np.all(np.isfinite(b)):
            scales[at] = 255
            continue
        top = float(np.abs(b).max())
        e = 1
        if top > 0:
            mant, exp = np.frexp(top)                    # top = mant 2^exp, mant in [0.5, 1)
            e = int(exp) - 1 - 2 + 127 + (1 if mant >= 0.875 else 0)
        e = min(252, max(1, e))
        scales[at] = e
        m = np.abs(b) / 2.0 ** (e - 127)
        dist = np.abs(m[:, None] - MAGNITUDES[None, :])
        # nearest, ties to the even code: among the nearest two the even one comes first
        order = np.array([0, 2, 4, 6, 1, 3, 5, 7])
        c = order[np.argmin(dist[:, order], axis=1)]
        codes[at] = c + 8 * np.signbit(b)
    return codes.reshape(x.shape), scales


def dequantize(codes, scales):
    mag = MAGNITUDES[codes & 7]
    unit = np.where(scales == 255, np.nan, np.exp2(scales.astype(np.float64) - 127))
    return np.where(codes >= 8, -mag, mag) * np.repeat(unit, 32, axis=-1)


def empty_cache(n_pages, page_size, heads, d, fill=0):
    return (np.full((n_pages, heads, page_size, d // 2), fill, np.uint8),
            np.full((n_pages, heads, page_size, d // 32), fill, np.uint8),
            np.full((n_pages, heads, page_size // 4, d // 8, 4, 4), fill, np.uint8),
            np.full((n_pages, heads, page_size // 4, d // 32, 4), fill, np.uint8))


def write(cache, k, v, slots):
    kc, ks, vc, vs = cache
    n_pages, heads, page, half = kc.shape
    for t, slot in enumerate(slots):
        if slot < 0 or slot >= n_pages * page:
            continue
        p, o = divmod(int(slot), page)
        for h in range(heads):
            for arr, x in ((0, k), (1, v)):
                c, s = quantize(x[t, h])
                by = c[0::2] | (c[1::2] << 4)
                if arr == 0:
                    kc[p, h, o], ks[p, h, o] = by, s
                else:
                    vc[p, h, o // 4, :, o % 4], vs[p, h, o // 4, :, o % 4] = by.reshape(-1, 4), s


def read(cache, slots):
    kc, ks, vc, vs = cache
    n_pages, heads, page, half = kc.shape
    out = [np.zeros((len(slots), heads, 2 * half)) for _ in range(2)]
    for t, slot in enumerate(slots):
        if slot < 0 or slot >= n_pages * page:
            continue
        p, o = divmod(int(slot), page)
        for i, (by, s) in enumerate(((kc[p, :, o], ks[p, :, o]),
                                     (vc[p, :, o // 4, :, o % 4].reshape(heads, half), vs[p, :, o // 4, :, o % 4]))):
            c = np.stack((by & 15, by >> 4), axis=-1).reshape(heads, 2 * half)
            out[i][t] = dequantize(c, s)
    return out


# ---------------------------------------------------------------- attention
def attention(q, cache, table, kv_len, q_start, scale, window=0):
    """(out, A, E), each [T, heads, d]: A = sum_t w_t |v_t|, and E = A (4 e + (L +
    d) 2^-24) bounds what fp32 sums leave: e is the largest rounding a score of d
    products can carry, L the number of tokens summed."""
    T, heads, d = q.shape
    page, kvh = cache[0].shape[2], cache[0].shape[1]
    out, mag, soft = np.zeros((T, heads, d)), np.zeros((T, heads, d)), np.zeros((T, heads, d))
    for b, L in enumerate(kv_len):
        L = int(L)
        q0, q1 = int(q_start[b]), int(q_start[b + 1])
        slots = [int(table[b][t // page]) * page + t % page for t in range(L)]
        K, V = read(cache, slots)
        for j in range(q1 - q0):
            P = L - (q1 - q0) + j
            lo = max(0, P - window + 1) if window else 0
            if P < lo:
                continue
            for h in range(heads):
                k, v = K[lo:P + 1, h // (heads // kvh)], V[lo:P + 1, h // (heads // kvh)]
                s = scale * (k @ q[q0 + j, h])
                e = (d + 8) * 2.0 ** -24 * scale * (np.abs(k) @ np.abs(q[q0 + j, h]))
                w = np.exp(s - s.max())
                w /= w.sum()
                out[q0 + j, h] = w @ v
                mag[q0 + j, h] = w @ np.abs(v)
                soft[q0 + j, h] = mag[q0 + j, h] * (4 * e.max() + (P + 1 - lo + d) * 2.0 ** -24)
    return out, mag, soft


# ---------------------------------------------------------------- norms, positions
def block_norm(x, weight, y=None, post=None, gate=None, scale=1.0, eps=1e-6):
    """(h, n, |x| + |scale gate u|)."""
    def unit(a):
        return a / np.sqrt((a * a).mean(axis=1, keepdims=True) + eps)
    h, mag = x, np.abs(x)
    if y is not None:
        u = y if post is None else unit(y) * post
        u = scale * (u if gate is None else u * gate)
        h, mag = x + u, mag + np.abs(u)
    return h, unit(h) * weight, mag


def rotary(x, cos, sin, positions, sections, interleaved=False):
    """(turned, |x1 cos| + |x2 sin| an element); positions [axes, T]."""
    out, mag = x.copy(), np.abs(x)
    half = cos.shape[1]
    axis = np.repeat(np.arange(len(sections)), sections)
    for t in range(x.shape[0]):
        for j in range(half):
            p = min(max(int(positions[axis[j]][t]), 0), cos.shape[0] - 1)
            c, s = float(cos[p, j]), float(sin[p, j])
            a, b = (2 * j, 2 * j + 1) if interleaved else (j, j + half)
            x1, x2 = x[t, :, a], x[t, :, b]
            out[t, :, a], out[t, :, b] = x1 * c - x2 * s, x2 * c + x1 * s
            mag[t, :, a], mag[t, :, b] = np.abs(x1 * c) + np.abs(x2 * s), np.abs(x2 * c) + np.abs(x1 * s)
    return out, mag
