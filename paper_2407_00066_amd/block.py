"""What a decoder block needs around its multi-adapter layers
(include/cts_block.h): the 4-bit key/value cache with its writes, reads and
attention (of trees of drafted tokens too), the norms with the residual, and rotary positions.

Argument marshalling only, like the layer's binding: every step runs in
libcts.so's kernels, on torch's current stream.  Head arrays [T, heads,
head_dim] may be slices of packed rows: heads and elements are contiguous, rows
may lie further apart.
"""
from __future__ import annotations

import ctypes

import torch

from . import _binding
from ._binding import AttnProblem, KvCacheArrays, _check, _check_tensor, _dev, _dt, _load_marshal, lib

U8, I32, I64, F32 = torch.uint8, torch.int32, torch.int64, torch.float32

# The calls are made natively (a decode step's take the GPU a few microseconds
# each); where one refuses an argument, the functions below find out which.
_native = _load_marshal()
_entries: dict = {}


def _entry(name: str) -> int:
    """The address of a C entry point."""
    at = _entries.get(name)
    if at is None:
        at = _entries[name] = ctypes.cast(getattr(lib(), name), ctypes.c_void_p).value
    return at


def _raw_stream(device: torch.device) -> int:
    # (a tensor's device has an index)
    return torch._C._cuda_getCurrentRawStream(device.index) if device.type == "cuda" else 0


def _refused(device: torch.device, where: str):
    """The checks of a call that was refused have found nothing wrong with its tensors."""
    if device.type != "cuda":
        raise ValueError("%s: tensors must be on a GPU, not on %s" % (where, device))
    raise ValueError("%s: arguments must be plain tensors and 32-bit sizes" % where)


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
        self._at = ctypes.addressof(self._c)

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
    dev = cache.device
    st = _native.kv_write(_entry("cts_kv_write"), _raw_stream(dev), dev, cache._at, k, v, slots)
    if st is None:
        _dt(k, "k")
        shape = (k.shape[0], cache.n_heads, cache.head_dim)
        _rows(k, "k", dev, k.dtype, shape)
        _rows(v, "v", dev, k.dtype, shape)
        _dev(slots, "slots", dev, I64, (shape[0],))
        _refused(dev, "kv_write")
    _check(st, "cts_kv_write")


def kv_read(cache: KVCache, slots, dtype=torch.bfloat16, k_out=None, v_out=None):
    """(k, v) [T, heads, head_dim]: what the cache holds for slots [T] (outside
    the cache: zeros).  See cts_kv_read."""
    dev = cache.device
    r = _native.kv_read(_entry("cts_kv_read"), _raw_stream(dev), dev, cache._at, slots, dtype, k_out, v_out)
    if r is None:
        shape = (slots.numel(), cache.n_heads, cache.head_dim)
        _dev(slots, "slots", dev, I64, (shape[0],))
        if k_out is not None:
            dtype = k_out.dtype
        _dt(torch.empty(0, dtype=dtype), "the output")
        for t, name in ((k_out, "k_out"), (v_out, "v_out")):
            if t is not None:
                _rows(t, name, dev, dtype, shape)
        _refused(dev, "kv_read")
    _check(r[2], "cts_kv_read")
    return r[0], r[1]


def kv_attention_workspace_size(q, cache: KVCache, B, max_q, max_kv, window=0) -> int:
    """Bytes of workspace kv_attention needs for queries like q of B sequences
    (0 for a call it would refuse)."""
    sizes = (q.shape[0], B, q.shape[1], max(1, -(-max_kv // cache.page_size)), max_q, max_kv, window)
    if not all(-2 ** 31 <= n < 2 ** 31 for n in sizes):
        return 0                                        # (ctypes would take their low 32 bits)
    p = AttnProblem(*sizes, _dt(q, "q"), 1.0)
    return int(lib().cts_kv_attention_workspace_size(ctypes.byref(p), ctypes.byref(cache._c)))


def kv_attention_plan(q, cache: KVCache, block_table, max_q, max_kv, window=0) -> tuple:
    """(how, few, pieces) of kv_attention for tensors like these, for tests and
    debugging: how in "whole", "by length", "runs" (see cts_kv_attention_plan)."""
    B, cols = block_table.shape
    p = AttnProblem(q.shape[0], B, q.shape[1], cols, max_q, max_kv, window, _dt(q, "q"), 1.0)
    out = (ctypes.c_int32 * 3)()
    _check(lib().cts_kv_attention_plan(ctypes.byref(p), ctypes.byref(cache._c), out), "cts_kv_attention_plan")
    return ("whole", "by length", "runs")[out[0]], out[1], out[2]


def kv_attention(q, cache: KVCache, block_table, kv_len, q_start=None, max_q=None, max_kv=None, scale=None, window=0,
                 out=None, workspace=None):
    """Causal attention of q [T, n_q_heads, head_dim] over the cached tokens of
    the sequences of block_table [B, max_pages] and kv_len [B] (int32); q_start
    [B + 1] (int32) gives each sequence's query rows, None one row each.  max_q
    and max_kv bound the queries of a sequence and kv_len (None: all rows of q, and
    what the table has room for; tight bounds choose faster kernels).  Rows that
    belong to no sequence, or lie past max_q in theirs, are not written: without
    `out` they hold whatever the new tensor's memory did.  scale None:
    head_dim^-1/2.  See cts_kv_attention."""
    dev = cache.device
    r = _native.kv_attention(_entry("cts_kv_attention"), _entry("cts_kv_attention_workspace_size"), _raw_stream(dev), dev,
                             cache._at, q, block_table, kv_len, q_start, max_q, max_kv,
                             cache.head_dim ** -0.5 if scale is None else scale, window, out, workspace)
    if r is None:
        _dt(q, "q")
        shape = (q.shape[0], q.shape[1], cache.head_dim)
        _rows(q, "q", dev, q.dtype, shape)
        if out is not None:
            _rows(out, "out", dev, q.dtype, shape)
        B, cols = block_table.shape
        _dev(block_table, "block_table", dev, I32, (B, cols))
        _dev(kv_len, "kv_len", dev, I32, (B,))
        if q_start is not None:
            _dev(q_start, "q_start", dev, I32, (B + 1,))
        if workspace is not None:
            _dev(_binding._workspace(dev, 0, workspace), "workspace", dev, U8)
        _refused(dev, "kv_attention")
    _check(r[1], "cts_kv_attention")
    return r[0]


def block_norm(x, weight, y=None, post_weight=None, gate=None, scale=1.0, eps=1e-6, h_out=None, n_out=None):
    """(h, n): h = x + scale * gate * u, u = N(y) * post_weight (or y), and
    n = N(h) * weight, N(a) = a / sqrt(mean(a^2) + eps) over a token's elements.
    x, y [T, d]; weights [d]; gate [d] or [T, d].  y None: h is x itself, n its
    norm.  h_out may be x or y.  See cts_block_norm."""
    dev = x.device
    r = _native.block_norm(_entry("cts_block_norm"), _raw_stream(dev), dev, x, weight, y, post_weight, gate, scale, eps,
                           h_out, n_out)
    if r is None:
        tdt = x.dtype
        _dt(x, "x")
        T, d = x.shape
        if y is None and not (post_weight is None and gate is None and h_out is None):
            raise ValueError("post_weight, gate and h_out go with y")
        for t, name in ((x, "x"), (y, "y"), (h_out, "h_out"), (n_out, "n_out")):
            if t is not None:
                _rows(t, name, dev, tdt, (T, d))
        for t, name in ((weight, "weight"), (post_weight, "post_weight")):
            if t is not None or name == "weight":
                _dev(t, name, dev, tdt, (d,))
        if gate is not None:
            if gate.dim() == 1:
                _dev(gate, "gate", dev, tdt, (d,))
            else:
                _rows(gate, "gate", dev, tdt, (T, d))
        _refused(dev, "block_norm")
    _check(r[2], "cts_block_norm")
    return (x if y is None else r[0]), r[1]


def _check_angles(dev, T, cos, sin, positions, sections):
    n_pos, half = cos.shape
    _dev(cos, "cos", dev, F32, (n_pos, half))
    _dev(sin, "sin", dev, F32, (n_pos, half))
    axes = 1 if positions.dim() == 1 else positions.shape[0]
    _dev(positions, "positions", dev, I32, (T,) if positions.dim() == 1 else (axes, T))
    if sections is not None and len(sections) != axes:
        raise ValueError("sections must hold a count for each of the %d axes" % axes)


def rotary(q, k, cos, sin, positions, sections=None, interleaved=False, q_out=None, k_out=None):
    """(q', k'): q [T, n_q_heads, head_dim] and k [T, n_k_heads, head_dim]
    (either may be None) turned by the angles of cos, sin (fp32 [n_pos, rot_dim / 2])
    at positions (int32 [n_axes, T], or [T]); sections: the pairs of each axis.
    q_out, k_out may be q, k.  See cts_rotary."""
    some = q if q is not None else k
    if some is None:
        raise ValueError("q or k is needed")
    dev = some.device
    r = _native.rotary(_entry("cts_rotary"), _raw_stream(dev), dev, q, k, cos, sin, positions, sections, interleaved, q_out,
                       k_out)
    if r is None:
        tdt = some.dtype
        _dt(some, "q")
        T, _, d = some.shape
        for t, o, name in ((q, q_out, "q"), (k, k_out, "k")):
            if t is None:
                if o is not None:
                    raise ValueError("%s_out goes with %s" % (name, name))
                continue
            shape = (T, t.shape[1], d)
            _rows(t, name, dev, tdt, shape)
            if o is not None:
                _rows(o, name + "_out", dev, tdt, shape)
        _check_angles(dev, T, cos, sin, positions, sections)
        _refused(dev, "rotary")
    _check(r[2], "cts_rotary")
    return r[0], r[1]


def kv_append(cache: KVCache, q, k, v, slots, cos, sin, positions, sections=None, interleaved=False, q_out=None, k_out=None):
    """q' = rotary(q), and kv_write of rotary(k) and v [T, heads, head_dim], in one
    launch and with the same bits; q (None: keys and values alone, and None is returned) is
    [T, n_q_heads, head_dim].  k_out receives the turned keys too (None: the cache
    alone does).  q_out, k_out may be q, k.  See rotary, kv_write and cts_kv_append."""
    dev = cache.device
    r = _native.kv_append(_entry("cts_kv_append"), _raw_stream(dev), dev, cache._at, q, k, v, slots, cos, sin, positions,
                          sections, interleaved, q_out, k_out)
    if r is None:
        _dt(k, "k")
        T, shape = k.shape[0], (k.shape[0], cache.n_heads, cache.head_dim)
        if q is None and q_out is not None:
            raise ValueError("q_out goes with q")
        for t, name in ((k, "k"), (v, "v"), (k_out, "k_out")):
            if t is not None or name != "k_out":
                _rows(t, name, dev, k.dtype, shape)
        for t, name in ((q, "q"), (q_out, "q_out")):
            if t is not None:
                _rows(t, name, dev, k.dtype, (T, q.shape[1], cache.head_dim))
        _dev(slots, "slots", dev, I64, (T,))
        _check_angles(dev, T, cos, sin, positions, sections)
        _refused(dev, "kv_append")
    _check(r[1], "cts_kv_append")
    return r[0]


def kv_tree_attention_workspace_size(q, cache: KVCache, B, max_q, max_kv, window=0) -> int:
    """Bytes of workspace kv_tree_attention needs for queries like q of B
    sequences (0 for a call it would refuse)."""
    sizes = (q.shape[0], B, q.shape[1], max(1, -(-max_kv // cache.page_size)), max_q, max_kv, window)
    if not all(-2 ** 31 <= n < 2 ** 31 for n in sizes):
        return 0
    p = AttnProblem(*sizes, _dt(q, "q"), 1.0)
    return int(lib().cts_kv_tree_attention_workspace_size(ctypes.byref(p), ctypes.byref(cache._c)))


def kv_tree_attention_plan(q, cache: KVCache, block_table, max_q, max_kv, window=0) -> tuple:
    """(rows, how, waves) of kv_tree_attention for tensors like these, for tests and
    debugging: how in "whole", "by work", "cut" (see cts_kv_tree_attention_plan)."""
    B, cols = block_table.shape
    p = AttnProblem(q.shape[0], B, q.shape[1], cols, max_q, max_kv, window, _dt(q, "q"), 1.0)
    out = (ctypes.c_int32 * 3)()
    _check(lib().cts_kv_tree_attention_plan(ctypes.byref(p), ctypes.byref(cache._c), out), "cts_kv_tree_attention_plan")
    return out[0], ("whole", "by work", "cut")[out[1]], out[2]


def kv_tree_attention(q, cache: KVCache, block_table, kv_len, mask, q_start=None, max_q=None, max_kv=None, scale=None,
                      window=0, positions=None, out=None, workspace=None):
    """Attention of drafted tokens q [T, n_q_heads, head_dim]: each sequence's rows
    are its last n cached tokens; a row sees the tokens before them (with a window, those
    less than that before positions [T], int32) and the drafts whose bits its
    mask [T, words] (int32, 32 drafts a word, the lowest bit first) has.  The rest
    as for kv_attention; max_q is at most 512, and the mask has a bit for each (None: all
    rows of q, refused where these are more).  See cts_kv_tree_attention."""
    dev = cache.device
    r = _native.kv_tree_attention(_entry("cts_kv_tree_attention"), _entry("cts_kv_tree_attention_workspace_size"),
                                  _raw_stream(dev), dev, cache._at, q, block_table, kv_len, mask, q_start, max_q, max_kv,
                                  cache.head_dim ** -0.5 if scale is None else scale, window, positions, out, workspace)
    if r is None:
        _dt(q, "q")
        shape = (q.shape[0], q.shape[1], cache.head_dim)
        _rows(q, "q", dev, q.dtype, shape)
        if out is not None:
            _rows(out, "out", dev, q.dtype, shape)
        B, cols = block_table.shape
        _dev(block_table, "block_table", dev, I32, (B, cols))
        _dev(kv_len, "kv_len", dev, I32, (B,))
        if not isinstance(mask, torch.Tensor) or mask.dim() != 2:
            raise ValueError("mask must be [T, words]")
        _dev(mask, "mask", dev, I32, (q.shape[0], mask.shape[1]))
        if q_start is not None:
            _dev(q_start, "q_start", dev, I32, (B + 1,))
        if positions is not None:
            _dev(positions, "positions", dev, I32, (q.shape[0],))
        if workspace is not None:
            _dev(_binding._workspace(dev, 0, workspace), "workspace", dev, U8)
        if max_q is None and q_start is not None and q.shape[0] > min(32 * mask.shape[1], 512):
            raise ValueError("max_q is needed: without it all %d rows may be one sequence's drafts, of which the mask has bits "
                             "for %d and a sequence at most 512" % (q.shape[0], 32 * mask.shape[1]))
        _refused(dev, "kv_tree_attention")
    _check(r[1], "cts_kv_tree_attention")
    return r[0]


def kv_keep(cache: KVCache, block_table, kv_len, q_start, path, n_path) -> None:
    """Keeps the accepted drafts: the last q_start[b + 1] - q_start[b] of sequence
    b's kv_len[b] cached tokens are drafts, and draft path[b, i] becomes the i-th of
    them for i < n_path[b] (path [B, max_path], n_path [B], int32).  The
    sequence's length is the caller's to set.  See cts_kv_keep."""
    dev = cache.device
    st = _native.kv_keep(_entry("cts_kv_keep"), _raw_stream(dev), dev, cache._at, block_table, kv_len, q_start, path, n_path)
    if st is None:
        B, cols = block_table.shape
        _dev(block_table, "block_table", dev, I32, (B, cols))
        _dev(kv_len, "kv_len", dev, I32, (B,))
        _dev(q_start, "q_start", dev, I32, (B + 1,))
        if not isinstance(path, torch.Tensor) or path.dim() != 2:
            raise ValueError("path must be [B, max_path]")
        _dev(path, "path", dev, I32, (B, path.shape[1]))
        _dev(n_path, "n_path", dev, I32, (B,))
        _refused(dev, "kv_keep")
    _check(st, "cts_kv_keep")
