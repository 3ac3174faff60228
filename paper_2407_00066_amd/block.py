"""What a decoder block needs around its multi-adapter layers
(include/cts_block.h): the 4-bit key/value cache with its writes, reads and
attention, the norms with the residual, and rotary positions.

Argument marshalling only, like the layer's binding: every step runs in
libcts.so's kernels, on torch's current stream.  Head arrays [T, heads,
head_dim] may be slices of packed rows: heads and elements are contiguous, rows
may lie further apart.
"""
from __future__ import annotations

import ctypes

import torch

from ._binding import AttnProblem, KvCacheArrays, _check, _check_tensor, _dev, _dt, _stream, _workspace, lib

U8, I32, I64, F32 = torch.uint8, torch.int32, torch.int64, torch.float32


class KVCache:
    """One layer's cache: four uint8 arrays in the layouts of cts_kv_cache,
      k_codes  [n_pages, heads, page_size, head_dim / 2]
      k_scales [n_pages, heads, page_size, head_dim / 32]
      v_codes  [n_pages, heads, page_size / 4, head_dim / 8, 4, 4]
      v_scales [n_pages, heads, page_size / 4, head_dim / 32, 4]
    (kv_cache allocates them).  The arrays' storage is the caller's; it must
    stay where it is while the object is used."""

    def __init__(self, k_codes, k_scales, v_codes, v_scales):
        if k_codes.dim() != 4:
            raise ValueError("k_codes must be [n_pages, heads, page_size, head_dim / 2]")
        n, h, s, half = k_codes.shape
        d = 2 * half
        self.device = dev = k_codes.device
        self.n_pages, self.n_heads, self.page_size, self.head_dim = n, h, s, d
        self.k_codes, self.k_scales, self.v_codes, self.v_scales = k_codes, k_scales, v_codes, v_scales
        at = [_dev(k_codes, "k_codes", dev, U8, (n, h, s, half)),
              _dev(k_scales, "k_scales", dev, U8, (n, h, s, d // 32)),
              _dev(v_codes, "v_codes", dev, U8, (n, h, s // 4, d // 8, 4, 4)),
              _dev(v_scales, "v_scales", dev, U8, (n, h, s // 4, d // 32, 4))]
        self._c = KvCacheArrays(n, s, h, d, *at)

    @property
    def n_slots(self) -> int:
        return self.n_pages * self.page_size


def kv_cache(n_pages, page_size, n_heads, head_dim, device="cuda") -> KVCache:
    """A cache of zeros."""
    def new(*shape):
        return torch.zeros(shape, dtype=U8, device=device)
    return KVCache(new(n_pages, n_heads, page_size, head_dim // 2), new(n_pages, n_heads, page_size, head_dim // 32),
                   new(n_pages, n_heads, page_size // 4, head_dim // 8, 4, 4),
                   new(n_pages, n_heads, page_size // 4, head_dim // 32, 4))


def _rows(t, name, device, dtype, shape):
    """(address, row stride) of an array [T, ...] whose rows are contiguous."""
    if not isinstance(t, torch.Tensor) or t.device != device or t.dtype != dtype or tuple(t.shape) != tuple(shape) \
            or t.layout != torch.strided:
        _check_tensor(t, name, device, dtype, shape)     # says what is wrong
        raise ValueError("%s must be a strided tensor of shape %s" % (name, tuple(shape)))
    width, strides = 1, t.stride()
    for n, s in zip(reversed(shape[1:]), reversed(strides[1:])):
        if s != width and n != 1:
            raise ValueError("%s must be contiguous within a row" % name)
        width *= n
    # (a single row's stride is arbitrary)
    return (t.data_ptr() if t.numel() else None), (strides[0] if shape[0] > 1 else width)


def kv_write(cache: KVCache, k, v, slots) -> None:
    """Quantises k, v [T, heads, head_dim] into the cache's slots [T] (int64,
    page * page_size + offset; outside the cache: skipped).  See cts_kv_write."""
    dev, T = cache.device, k.shape[0]
    shape = (T, cache.n_heads, cache.head_dim)
    dt = _dt(k, "k")
    kp, ldk = _rows(k, "k", dev, k.dtype, shape)
    vp, ldv = _rows(v, "v", dev, k.dtype, shape)
    _check(lib().cts_kv_write(ctypes.byref(cache._c), T, kp, ldk, vp, ldv, _dev(slots, "slots", dev, I64, (T,)), dt,
                              _stream(dev)), "cts_kv_write")


def kv_read(cache: KVCache, slots, dtype=torch.bfloat16, k_out=None, v_out=None):
    """(k, v) [T, heads, head_dim]: what the cache holds for slots [T] (outside
    the cache: zeros).  See cts_kv_read."""
    dev, T = cache.device, slots.numel()
    shape = (T, cache.n_heads, cache.head_dim)
    k = torch.empty(shape, dtype=dtype, device=dev) if k_out is None else k_out
    v = torch.empty(shape, dtype=k.dtype, device=dev) if v_out is None else v_out
    dt = _dt(k, "k_out")
    kp, ldk = _rows(k, "k_out", dev, k.dtype, shape)
    vp, ldv = _rows(v, "v_out", dev, k.dtype, shape)
    _check(lib().cts_kv_read(ctypes.byref(cache._c), T, _dev(slots, "slots", dev, I64, (T,)), kp, ldk, vp, ldv, dt,
                             _stream(dev)), "cts_kv_read")
    return k, v


def _attn_problem(q, cache, B, max_pages, max_q, max_kv, window, scale):
    T, heads = q.shape[0], q.shape[1]
    return AttnProblem(T, B, heads, max_pages, max_q, max_kv, window, _dt(q, "q"),
                       cache.head_dim ** -0.5 if scale is None else scale)


def kv_attention_workspace_size(q, cache: KVCache, B, max_q, max_kv, window=0) -> int:
    """Bytes of workspace kv_attention needs for queries like q of B sequences
    (0 for a call it would refuse)."""
    p = _attn_problem(q, cache, B, max(1, -(-max_kv // cache.page_size)), max_q, max_kv, window, 1.0)
    return int(lib().cts_kv_attention_workspace_size(ctypes.byref(p), ctypes.byref(cache._c)))


def kv_attention(q, cache: KVCache, block_table, kv_len, q_start=None, max_q=1, max_kv=None, scale=None, window=0,
                 out=None, workspace=None):
    """Causal attention of q [T, n_q_heads, head_dim] over the cached tokens of
    the sequences of block_table [B, max_pages] and kv_len [B] (int32); q_start
    [B + 1] (int32) gives each sequence's query rows, None one row each.  max_q
    and max_kv bound the queries of a sequence and kv_len (max_kv None: what the
    table has room for).  scale None: head_dim^-1/2.  See cts_kv_attention."""
    dev = cache.device
    T, heads = q.shape[0], q.shape[1]
    B, max_pages = block_table.shape
    shape = (T, heads, cache.head_dim)
    qp, ldq = _rows(q, "q", dev, q.dtype, shape)
    if out is None:
        out = torch.empty(shape, dtype=q.dtype, device=dev)
    op, ldo = _rows(out, "out", dev, q.dtype, shape)
    p = _attn_problem(q, cache, B, max_pages, max_q, max_pages * cache.page_size if max_kv is None else max_kv, window,
                      scale)
    c = ctypes.byref(cache._c)
    args = (_dev(block_table, "block_table", dev, I32, (B, max_pages)), _dev(kv_len, "kv_len", dev, I32, (B,)),
            None if q_start is None else _dev(q_start, "q_start", dev, I32, (B + 1,)))
    ws = _workspace(dev, int(lib().cts_kv_attention_workspace_size(ctypes.byref(p), c)) if workspace is None else 0,
                    workspace)
    _check(lib().cts_kv_attention(ctypes.byref(p), c, qp, ldq, *args, op, ldo, ws.data_ptr(), ws.numel(),
                                  _stream(dev)), "cts_kv_attention")
    return out


def block_norm(x, weight, y=None, post_weight=None, gate=None, scale=1.0, eps=1e-6, h_out=None, n_out=None):
    """(h, n): h = x + scale * gate * u, u = N(y) * post_weight (or y), and
    n = N(h) * weight, N(a) = a / sqrt(mean(a^2) + eps) over a token's elements.
    x, y [T, d]; weights [d]; gate [d] or [T, d].  y None: h is x itself, n its
    norm.  h_out may be x or y.  See cts_block_norm."""
    dev, (T, d) = x.device, x.shape
    dt, tdt = _dt(x, "x"), x.dtype
    xp, ldx = _rows(x, "x", dev, tdt, (T, d))
    wp = _dev(weight, "weight", dev, tdt, (d,))
    yp = pp = gp = hp = None
    ldy = ldg = ldh = 0
    h = x
    if y is not None:
        yp, ldy = _rows(y, "y", dev, tdt, (T, d))
        if post_weight is not None:
            pp = _dev(post_weight, "post_weight", dev, tdt, (d,))
        if gate is not None:
            if gate.dim() == 1:
                gp = _dev(gate, "gate", dev, tdt, (d,))
            else:
                gp, ldg = _rows(gate, "gate", dev, tdt, (T, d))
        h = torch.empty((T, d), dtype=tdt, device=dev) if h_out is None else h_out
        hp, ldh = _rows(h, "h_out", dev, tdt, (T, d))
    elif post_weight is not None or gate is not None or h_out is not None:
        raise ValueError("post_weight, gate and h_out go with y")
    n = torch.empty((T, d), dtype=tdt, device=dev) if n_out is None else n_out
    np_, ldn = _rows(n, "n_out", dev, tdt, (T, d))
    _check(lib().cts_block_norm(T, d, dt, xp, ldx, yp, ldy, pp, gp, ldg, float(scale), float(eps), wp, hp, ldh, np_, ldn,
                                _stream(dev)), "cts_block_norm")
    return h, n


def rotary(q, k, cos, sin, positions, sections=None, interleaved=False, q_out=None, k_out=None):
    """(q', k'): q [T, n_q_heads, head_dim] and k [T, n_k_heads, head_dim]
    (either may be None) turned by the angles of cos, sin (fp32 [n_pos, rot_dim / 2])
    at positions (int32 [n_axes, T], or [T]); sections: the pairs of each axis.
    q_out, k_out may be q, k.  See cts_rotary."""
    some = q if q is not None else k
    if some is None:
        raise ValueError("q or k is needed")
    dev, tdt, T, d = some.device, some.dtype, some.shape[0], some.shape[2]
    dt = _dt(some, "q")
    n_pos, half = cos.shape
    n_axes = 1 if positions.dim() == 1 else positions.shape[0]
    args, outs, heads = [], [], []
    for t, o, name in ((q, q_out, "q"), (k, k_out, "k")):
        if t is None:
            if o is not None:
                raise ValueError("%s_out goes with %s" % (name, name))
            args.append((None, 0, None, 0))
            outs.append(None)
            heads.append(0)
            continue
        shape = (T, t.shape[1], d)
        o = torch.empty(shape, dtype=tdt, device=dev) if o is None else o
        args.append(_rows(t, name, dev, tdt, shape) + _rows(o, name + "_out", dev, tdt, shape))
        outs.append(o)
        heads.append(t.shape[1])
    if sections is not None and len(sections) != n_axes:
        raise ValueError("sections must hold a count for each of the %d axes" % n_axes)
    sec = None if sections is None else (ctypes.c_int32 * n_axes)(*[int(s) for s in sections])
    (qp, ldq, qo, ldqo), (kp, ldk, ko, ldko) = args
    _check(lib().cts_rotary(T, heads[0], heads[1], d, 2 * half, dt, qp, ldq, kp, ldk,
                            _dev(cos, "cos", dev, F32, (n_pos, half)), _dev(sin, "sin", dev, F32, (n_pos, half)), n_pos,
                            _dev(positions, "positions", dev, I32, (T,) if positions.dim() == 1 else (n_axes, T)), n_axes,
                            sec, int(bool(interleaved)), qo, ldqo, ko, ldko, _stream(dev)), "cts_rotary")
    return outs[0], outs[1]
