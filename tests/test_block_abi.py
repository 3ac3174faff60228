"""Argument checks of include/cts_block.h: every error is found on the host
before any HIP call (CPU; no call here reaches a kernel launch)."""
import ctypes

import pytest
import torch

import paper_2407_00066_amd as cts
from paper_2407_00066_amd import _binding as B
from paper_2407_00066_amd import block

INVALID, UNSUPPORTED, OK, WORKSPACE = B.CTS_ERR_INVALID_ARG, B.CTS_ERR_UNSUPPORTED, B.CTS_OK, B.CTS_ERR_WORKSPACE
BASE = 0x5000_0000_0000


def far(i, off=0):
    """Addresses a terabyte apart, never dereferenced."""
    return BASE + (i << 40) + off


def _cache(**kw):
    d = dict(n_pages=8, page_size=16, n_heads=2, head_dim=64, k_codes=far(0), k_scales=far(1), v_codes=far(2),
             v_scales=far(3))
    d.update(kw)
    return B.KvCacheArrays(**d)


BAD_CACHES = [(dict(n_pages=0), INVALID), (dict(page_size=-16), INVALID), (dict(n_heads=0), INVALID),
              (dict(head_dim=0), INVALID), (dict(page_size=8), UNSUPPORTED), (dict(page_size=48), UNSUPPORTED),
              (dict(page_size=2048), UNSUPPORTED), (dict(head_dim=96), UNSUPPORTED), (dict(n_heads=4097), UNSUPPORTED)]
BAD_ARRAYS = [dict(k_codes=0), dict(v_scales=0), dict(v_codes=far(2, 8)), dict(k_scales=far(1, 1)),
              dict(v_codes=far(0, 64)), dict(v_scales=far(1))]


def _write(c=None, T=3, k=far(5), ldk=128, v=far(6), ldv=128, slots=far(7), dtype=B.CTS_BF16, read=False):
    c = _cache() if c is None else c
    if read:
        return cts.lib().cts_kv_read(ctypes.byref(c), T, slots, k, ldk, v, ldv, dtype, None)
    return cts.lib().cts_kv_write(ctypes.byref(c), T, k, ldk, v, ldv, slots, dtype, None)


@pytest.mark.parametrize("read", [False, True])
def test_kv_calls_refuse(read):
    for kw, code in BAD_CACHES:
        assert _write(_cache(**kw), read=read) == code, kw
        assert _write(_cache(**kw), T=0, read=read) == code, kw
    for kw in BAD_ARRAYS:
        assert _write(_cache(**kw), read=read) == INVALID, kw
    for kw, code in [(dict(T=-1), INVALID), (dict(k=0), INVALID), (dict(v=0), INVALID), (dict(slots=0), INVALID),
                     (dict(k=far(5, 8)), INVALID), (dict(slots=far(7, 4)), INVALID), (dict(ldk=127), INVALID),
                     (dict(ldv=132), INVALID), (dict(ldk=-128), INVALID), (dict(ldk=1 << 40), INVALID),
                     (dict(dtype=2), UNSUPPORTED), (dict(k=far(0, 32)), INVALID), (dict(v=far(3)), INVALID),
                     (dict(slots=far(2)), INVALID)]:
        assert _write(read=read, **kw) == code, kw
    assert _write(T=0, k=0, v=0, slots=0, read=read) == OK


def test_kv_read_outputs_meet():
    assert _write(read=True, v=far(5)) == INVALID
    assert _write(read=True, v=far(5, 128), ldk=256, ldv=256) == INVALID      # 64 columns of both
    assert _write(read=True, slots=far(5, 16)) == INVALID
    assert cts.lib().cts_kv_read(None, 1, far(7), far(5), 128, far(6), 128, 1, None) == INVALID


def _problem(**kw):
    d = dict(T=4, B=4, n_q_heads=4, max_pages=3, max_q=1, max_kv=40, window=0, dtype=B.CTS_BF16, scale=0.125)
    d.update(kw)
    return B.AttnProblem(**d)


def _attend(p=None, c=None, q=far(5), ldq=256, table=far(6), kv_len=far(7), q_start=None, out=far(8), ldo=256, ws=far(9),
            ws_bytes=1 << 36):
    p = _problem() if p is None else p
    c = _cache() if c is None else c
    return cts.lib().cts_kv_attention(ctypes.byref(p), ctypes.byref(c), q, ldq, table, kv_len, q_start, out, ldo, ws,
                                      ws_bytes, None)


@pytest.mark.parametrize("kw,code", [
    (dict(T=-1), INVALID), (dict(B=-1), INVALID), (dict(n_q_heads=0), INVALID), (dict(n_q_heads=3), INVALID),
    (dict(max_pages=0), INVALID), (dict(max_q=0), INVALID), (dict(max_kv=-1), INVALID), (dict(window=-1), INVALID),
    (dict(scale=0.0), INVALID), (dict(scale=-1.0), INVALID), (dict(scale=float("nan")), INVALID),
    (dict(scale=float("inf")), INVALID), (dict(dtype=3), UNSUPPORTED), (dict(n_q_heads=65538), UNSUPPORTED),
    (dict(max_q=1 << 25), UNSUPPORTED), (dict(max_kv=2 ** 31 - 1), UNSUPPORTED),
    (dict(B=2 ** 31 - 1, T=2 ** 31 - 1), UNSUPPORTED), (dict(T=5), INVALID), (dict(max_q=2), INVALID)])
def test_attention_refuses_problems(kw, code):
    assert _attend(_problem(**kw)) == code
    if code == UNSUPPORTED:
        p, c = _problem(**kw), _cache()
        assert cts.lib().cts_kv_attention_workspace_size(ctypes.byref(p), ctypes.byref(c)) == 0


def test_attention_refuses_arguments():
    for kw, code in BAD_CACHES:
        assert _attend(c=_cache(**kw)) == code, kw
    for kw in BAD_ARRAYS:
        assert _attend(c=_cache(**kw)) == INVALID, kw
    for kw in [dict(q=0), dict(q=far(5, 8)), dict(ldq=255), dict(ldq=260), dict(table=0), dict(table=far(6, 2)),
               dict(kv_len=0), dict(kv_len=far(7, 1)), dict(q_start=far(10, 2)), dict(out=0), dict(out=far(8, 4)),
               dict(ldo=8), dict(ws=0), dict(ws=far(9, 8)), dict(out=far(5)), dict(out=far(0)), dict(out=far(6, 16)),
               dict(ws=far(5, 256)), dict(ws=far(8)), dict(ws=far(2)), dict(q_start=far(8, 16)),
               dict(ws=far(7) - (1 << 30), ws_bytes=1 << 31)]:
        assert _attend(**kw) == INVALID, kw
    assert cts.lib().cts_kv_attention(None, ctypes.byref(_cache()), *[far(5), 256, far(6), far(7), None, far(8), 256,
                                                                      far(9), 1 << 30, None]) == INVALID


def test_attention_workspace():
    c, p = _cache(), _problem()
    need = cts.lib().cts_kv_attention_workspace_size(ctypes.byref(p), ctypes.byref(c))
    assert need > 0 and _attend(ws_bytes=need - 1) == WORKSPACE
    assert _attend(_problem(T=0, B=0), q=0, table=0, kv_len=0, out=0, ws=0, ws_bytes=0) == OK


def test_attention_workspace_does_not_fall():
    """A workspace for the largest batch serves every smaller one; a window never needs more."""
    def need(B_, max_q, max_kv, window=0, heads=8, kvh=2, d=128, dtype=B.CTS_BF16):
        c = _cache(n_heads=kvh, head_dim=d, n_pages=1 << 20)
        p = _problem(T=B_ * max_q, B=B_, n_q_heads=heads, max_q=max_q, max_kv=max_kv, window=window, max_pages=1 << 16,
                     dtype=dtype)
        return cts.lib().cts_kv_attention_workspace_size(ctypes.byref(p), ctypes.byref(c))
    sizes = [0, 1, 2, 3, 5, 8, 16, 31, 33, 64, 100, 127, 129, 500, 2000]
    for dtype in (B.CTS_BF16, B.CTS_F32):
        for d in (64, 128, 256):
            for fixed in (1, 7, 64, 300):
                rows = [need(n, fixed, 4000, d=d, dtype=dtype) for n in sizes]
                assert rows == sorted(rows)
                rows = [need(fixed, max(n, 1), 4000, d=d, dtype=dtype) for n in sizes]
                assert rows == sorted(rows)
                rows = [need(fixed, 3, 37 * n, d=d, dtype=dtype) for n in sizes]
                assert rows == sorted(rows)
                assert all(need(fixed, 9, 5000, w, d=d, dtype=dtype) <= need(fixed, 9, 5000, d=d, dtype=dtype)
                           for w in (1, 50, 700, 5000, 9000))


def _norm(T=3, d=64, dtype=B.CTS_BF16, x=far(0), ldx=64, y=far(1), ldy=64, post=far(2), gate=far(3), ldg=64, scale=1.0,
          eps=1e-6, w=far(4), h=far(5), ldh=64, n=far(6), ldn=64):
    return cts.lib().cts_block_norm(T, d, dtype, x, ldx, y, ldy, post, gate, ldg, scale, eps, w, h, ldh, n, ldn, None)


def test_norm_refuses():
    for kw, code in [(dict(T=-1), INVALID), (dict(d=0), INVALID), (dict(d=32769), UNSUPPORTED), (dict(dtype=5), UNSUPPORTED),
                     (dict(x=0), INVALID), (dict(w=0), INVALID), (dict(n=0), INVALID), (dict(h=0), INVALID),
                     (dict(x=far(0, 1)), INVALID), (dict(ldx=63), INVALID), (dict(ldy=1), INVALID), (dict(ldg=3), INVALID),
                     (dict(ldh=-64), INVALID), (dict(ldn=1 << 50), INVALID), (dict(scale=float("nan")), INVALID),
                     (dict(scale=float("inf")), INVALID), (dict(eps=-1.0), INVALID), (dict(eps=float("nan")), INVALID),
                     (dict(eps=float("inf")), INVALID), (dict(post=far(2, 1)), INVALID), (dict(gate=far(3, 1)), INVALID),
                     (dict(h=far(6)), INVALID), (dict(h=far(0, 2)), INVALID), (dict(h=far(0), ldh=128), INVALID),
                     (dict(n=far(1, 64)), INVALID), (dict(h=far(3)), INVALID), (dict(h=far(4)), INVALID),
                     (dict(n=far(2, 2)), INVALID), (dict(y=0), INVALID), (dict(y=0, post=0, gate=0), INVALID)]:
        assert _norm(**kw) == code, kw
    assert _norm(T=0, x=0, y=0, post=0, gate=0, w=0, h=0, n=0) == OK


def _rotary(T=3, hq=4, hk=2, d=64, rot=64, dtype=B.CTS_BF16, q=far(0), ldq=256, k=far(1), ldk=128, cos=far(2), sin=far(3),
            n_pos=10, pos=far(4), axes=1, sections=None, qo=far(5), ldqo=256, ko=far(6), ldko=128):
    sec = None if sections is None else (ctypes.c_int32 * len(sections))(*sections)
    return cts.lib().cts_rotary(T, hq, hk, d, rot, dtype, q, ldq, k, ldk, cos, sin, n_pos, pos, axes, sec, 0, qo, ldqo, ko,
                                ldko, None)


def test_rotary_refuses():
    for kw, code in [(dict(T=-1), INVALID), (dict(hq=-1), INVALID), (dict(hq=0, hk=0), INVALID), (dict(d=0), INVALID),
                     (dict(rot=0), INVALID), (dict(rot=80), INVALID), (dict(n_pos=0), INVALID), (dict(axes=0), INVALID),
                     (dict(axes=2), INVALID), (dict(axes=5, sections=[8, 8, 8, 4, 4]), UNSUPPORTED),
                     (dict(axes=2, sections=[16, 15]), INVALID), (dict(axes=2, sections=[33, -1]), INVALID),
                     (dict(axes=2, sections=[2 ** 31 - 1, 2 ** 31 - 1]), INVALID), (dict(rot=24), UNSUPPORTED),
                     (dict(d=72, rot=64), UNSUPPORTED), (dict(d=8192), UNSUPPORTED), (dict(dtype=9), UNSUPPORTED),
                     (dict(q=0), INVALID), (dict(ko=0), INVALID), (dict(q=far(0, 8)), INVALID), (dict(ldq=255), INVALID),
                     (dict(ldko=100), INVALID), (dict(cos=0), INVALID), (dict(sin=far(3, 4)), INVALID), (dict(pos=0), INVALID),
                     (dict(pos=far(4, 2)), INVALID), (dict(qo=far(6)), INVALID), (dict(qo=far(0, 16)), INVALID),
                     (dict(qo=far(1)), INVALID), (dict(ko=far(0)), INVALID), (dict(ko=far(2)), INVALID),
                     (dict(qo=far(4)), INVALID), (dict(qo=far(0), ldqo=512), INVALID)]:
        assert _rotary(**kw) == code, kw
    assert _rotary(T=0, q=0, k=0, cos=0, sin=0, pos=0, qo=0, ko=0) == OK


# ---------------------------------------------------------------- the Python side
def test_binding_checks_tensors():
    """Shapes, types, devices and strides (CPU tensors: nothing can be launched)."""
    cache = cts.kv_cache(2, 16, 2, 64, device="cpu")
    assert cache.n_slots == 32 and cache.head_dim == 64
    k = torch.zeros(3, 2, 64, dtype=torch.bfloat16)
    slots = torch.zeros(3, dtype=torch.int64)
    with pytest.raises(ValueError):
        cts.kv_write(cache, k[:, :1], k, slots)
    with pytest.raises(ValueError):
        cts.kv_write(cache, k, k.transpose(0, 1).contiguous().transpose(0, 1)[:, :, :], slots)
    with pytest.raises(TypeError):
        cts.kv_write(cache, k, k.float(), slots)
    with pytest.raises(TypeError):
        cts.kv_write(cache, k, k, slots.int())
    with pytest.raises(TypeError):
        cts.kv_write(cache, k.half(), k.half(), slots)
    with pytest.raises(ValueError):
        cts.kv_write(cache, k, k, slots[:2])
    with pytest.raises(TypeError):
        cts.kv_read(cache, slots, dtype=torch.float16)
    with pytest.raises(ValueError):
        cts.KVCache(cache.k_codes, cache.k_scales[:1], cache.v_codes, cache.v_scales)
    with pytest.raises(TypeError):
        cts.KVCache(cache.k_codes.float(), cache.k_scales, cache.v_codes, cache.v_scales)
    with pytest.raises(ValueError):
        cts.block_norm(torch.zeros(2, 8), torch.ones(8), gate=torch.ones(8))
    with pytest.raises(ValueError):
        cts.block_norm(torch.zeros(2, 8), torch.ones(7))
    with pytest.raises(ValueError):
        cts.rotary(None, None, torch.zeros(2, 8), torch.zeros(2, 8), torch.zeros(1, dtype=torch.int32))
    with pytest.raises(ValueError):
        cts.rotary(k, None, torch.zeros(2, 32), torch.zeros(2, 32), torch.zeros(3, dtype=torch.int32), sections=[16, 16])


def test_row_strides():
    t = torch.zeros(4, 6, 32)
    dev = t.device
    assert block._rows(t[:, 1:3], "t", dev, torch.float32, (4, 2, 32)) == (t.data_ptr() + 128, 192)
    assert block._rows(t[:1, 1:3], "t", dev, torch.float32, (1, 2, 32))[1] == 64
    assert block._rows(t[:, 1:2], "t", dev, torch.float32, (4, 1, 32))[1] == 192
    with pytest.raises(ValueError):
        block._rows(t[:, ::2], "t", dev, torch.float32, (4, 3, 32))
    with pytest.raises(ValueError):
        block._rows(t[..., ::2], "t", dev, torch.float32, (4, 6, 16))
    with pytest.raises(ValueError):
        block._rows(t[:1].expand(4, 6, 32)[:, :, :], "t", dev, torch.float32, (4, 6, 33))
