"""Sizes at which the decoder block's memory-bound operators take other kernels or
launches than in the small tests: streaming stores (outputs of 4 MB and more),
angles shared by several heads, several tokens a workgroup, and more rows than one
launch has threads for."""
import numpy as np
import pytest
import torch

import paper_2407_00066_amd as cts
from oracle import block as ob

from _block_helpers import ROUND, TORCH, assert_within, f64, to_device, to_host, values
from _gpu_helpers import say
from test_gpu_block_ops import EPS32, _check_norm, _norm_case

pytestmark = pytest.mark.gpu
MB4 = 4 << 20


def test_norm_of_more_rows_than_a_launch():
    """2^32 threads is what a launch cannot have: short rows reach it with 134 MB."""
    T = 2 ** 26 + 5
    x = torch.randn(T, 1, device="cuda").bfloat16()
    w = torch.full((1,), 3.0, dtype=torch.bfloat16, device="cuda")
    say("block_norm T=%d d=1" % T)
    n = torch.full_like(x, float("nan"))
    cts.block_norm(x, w, eps=1e-3, n_out=n)
    torch.cuda.synchronize()
    for at in range(0, T, 2 ** 24):
        a = x[at:at + 2 ** 24].float()
        want = 3 * a / (a * a + 1e-3).sqrt()
        # one rounding to bf16, and a few of fp32 on either side
        assert bool(((n[at:at + 2 ** 24].float() - want).abs() <= 1.001 * 2.0 ** -8 * want.abs()).all())


def test_block_norm_of_more_rows_than_a_launch():
    """With the residual, a gate for every token and outputs in place."""
    T, d = 2 ** 22 + 9, 2
    x, y, gate = (torch.randn(T, d, device="cuda") for _ in range(3))
    w, post = torch.tensor([3.0, -1.0], device="cuda"), torch.tensor([0.5, 2.0], device="cuda")

    def unit(a):
        return a / ((a * a).mean(1, keepdim=True) + 1e-3).sqrt()
    h = x.double() + 0.7 * gate.double() * unit(y.double()) * post.double()
    n = unit(h) * w.double()
    # h of two terms of a few roundings each; n's mean follows h's error
    mag = 8 * 2.0 ** -24 * (x.double().abs() + (0.7 * gate * post).double().abs() * 2)
    say("block_norm T=%d d=%d" % (T, d))
    got = cts.block_norm(x, w, y=y, post_weight=post, gate=gate, scale=0.7, eps=1e-3, h_out=x, n_out=y)
    assert got[0].data_ptr() == x.data_ptr()
    assert bool(((got[0].double() - h).abs() <= mag).all())
    rs = 1 / ((h * h).mean(1, keepdim=True) + 1e-3).sqrt()
    assert bool(((got[1].double() - n).abs() <= 3 * rs * (mag + mag.amax(1, keepdim=True) * n.abs()) + 2.0 ** -20 * n.abs()).all())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,d,post,gate,block", [(2101, 1032, True, "token", True), (2050, 1024, False, "channel", True),
                                                 (1100, 4104, True, "", True), (600, 9000, True, "channel", True),
                                                 (2099, 2000, False, "", False), (2301, 1033, True, "token", True)])
def test_norm_past_streaming_stores(T, d, post, gate, block, dtype):
    c = _norm_case(T, d, dtype, post, gate, block, T + d)
    assert (2 if block else 1) * c["x"][1].numel() * c["x"][1].element_size() >= MB4
    g = {k: (v[1] if v is not None else None) for k, v in c.items()}
    h_out, n_out = (torch.full((T + 2, d), 7.0, dtype=TORCH[dtype], device="cuda") for _ in range(2))
    say("block_norm %s T=%d d=%d" % (dtype, T, d))
    h, n = cts.block_norm(g["x"], g["weight"], y=g.get("y"), post_weight=g.get("post"), gate=g.get("gate"), scale=0.7,
                          eps=1e-5, h_out=h_out[1:-1] if block else None, n_out=n_out[1:-1])
    _check_norm(c, h, n, 0.7, 1e-5, dtype)
    for o in (h_out, n_out) if block else (n_out,):
        assert bool((o[[0, -1]] == 7).all())


def _turned(x, cos, sin, pos, sections, inter):
    """ob.rotary, all tokens at once."""
    half = cos.shape[1]
    axis, j = np.repeat(np.arange(len(sections)), sections), np.arange(half)
    p = np.clip(pos[axis].T, 0, cos.shape[0] - 1)                        # [T, half]
    c, s = (t.astype(np.float64)[p, j][:, None] for t in (cos, sin))
    a, b = (slice(0, 2 * half, 2), slice(1, 2 * half, 2)) if inter else (slice(0, half), slice(half, 2 * half))
    out, mag = x.copy(), np.abs(x)
    x1, x2 = x[..., a], x[..., b]
    out[..., a], out[..., b] = x1 * c - x2 * s, x2 * c + x1 * s
    mag[..., a], mag[..., b] = np.abs(x1 * c) + np.abs(x2 * s), np.abs(x2 * c) + np.abs(x1 * s)
    return out, mag


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("heads,kvh,d,rot,sections,inter", [
    (5, 2, 128, 128, [21, 22, 21], False), (3, 2, 64, 32, None, True), (4, 1, 256, 128, [30, 34], True), (1, 0, 128, 64, None, False),
    (2, 4, 64, 64, [3, 8, 10, 11], False)])
def test_rotary_with_shared_angles(heads, kvh, d, rot, sections, inter, dtype):
    """Four heads a thread, with a number of heads that is no multiple of four among them."""
    all_ = heads + kvh
    T = 2 ** 20 // (all_ * d // 16) + 7                                  # just past the switch
    rng = np.random.default_rng(d + heads)
    axes = len(sections) if sections else 1
    ang = rng.uniform(0, 100, (333, rot // 2))
    cos, sin = np.cos(ang).astype(np.float32), np.sin(ang).astype(np.float32)
    pos = rng.integers(-3, 340, (axes, T)).astype(np.int32)
    rows64, rows = values(rng, (T, (all_ + 1) * d), dtype)
    dc, ds, dp = torch.from_numpy(cos).cuda(), torch.from_numpy(sin).cuda(), torch.from_numpy(pos).cuda()
    q = rows[:, :heads * d].unflatten(1, (heads, d))
    k = rows[:, heads * d:all_ * d].unflatten(1, (kvh, d)) if kvh else None
    say("rotary %s T=%d heads=%d+%d d=%d" % (dtype, T, heads, kvh, d))
    got = cts.rotary(q, k, dc, ds, dp, sections=sections, interleaved=inter)
    want, mag = _turned(rows64[:, :all_ * d].reshape(T, all_, d), cos, sin, pos, sections or [rot // 2], inter)
    bound = 1.01 * ROUND[dtype] * np.abs(want) + 3 * EPS32 * mag
    for t, lo, hi in ((got[0], 0, heads), (got[1], heads, all_)):
        if t is not None:
            assert_within(t, want[:, lo:hi], bound[:, lo:hi], "rotary")
            assert np.array_equal(f64(t)[..., rot:], rows64[:, lo * d:hi * d].reshape(T, hi - lo, d)[..., rot:])
    before = rows[:, all_ * d:].clone()
    cts.rotary(q, k, dc, ds, dp, sections=sections, interleaved=inter, q_out=q, k_out=k)
    assert torch.equal(q, got[0]) and (k is None or torch.equal(k, got[1])) and torch.equal(rows[:, all_ * d:], before)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,heads,d,page", [(2053, 1, 64, 64), (1025, 3, 128, 16), (3077, 2, 64, 32), (5003, 1, 256, 128)])
def test_cache_of_several_tokens_a_workgroup(T, heads, d, page, dtype):
    """More than 1024 tokens: a workgroup's pieces belong to several, the last one's to fewer."""
    rng = np.random.default_rng(T)
    pages = -(-T // page) + 2
    slots = rng.permutation(pages * page)[:T].astype(np.int64)
    slots[rng.integers(0, T, 20)] = -1                                   # padding among them
    rows64, rows = values(rng, (T, (2 * heads + 1) * d), dtype)
    k64, v64 = (rows64[:, a * d:(a + heads) * d].reshape(T, heads, d) for a in (0, heads))
    k, v = (rows[:, a * d:(a + heads) * d].unflatten(1, (heads, d)) for a in (0, heads))
    host = ob.empty_cache(pages, page, heads, d, fill=37)
    cache = to_device(host)
    ds = torch.from_numpy(slots).cuda()
    say("kv_write %s T=%d heads=%d d=%d" % (dtype, T, heads, d))
    cts.kv_write(cache, k, v, ds)
    ob.write(host, k64, v64, slots)
    for got, want, name in zip(to_host(cache), host, ("k_codes", "k_scales", "v_codes", "v_scales")):
        assert np.array_equal(got, want), name
    for out in ("bf16", "f32"):
        gk, gv = (torch.full((T + 2, heads, d), 7.0, dtype=TORCH[out], device="cuda") for _ in range(2))
        cts.kv_read(cache, ds, k_out=gk[1:-1], v_out=gv[1:-1])
        for got, want in zip((gk, gv), ob.read(host, slots)):
            assert np.array_equal(f64(got[1:-1]), want) and bool((got[[0, -1]] == 7).all())


@pytest.mark.parametrize("out", ["bf16", "f32"])
def test_read_past_streaming_stores(out):
    """All slots of a cache of random bytes, 13 MB and more of them."""
    rng = np.random.default_rng(3)
    host = ob.empty_cache(65, 64, 3, 256)
    for a in (host[0], host[2]):
        a[...] = rng.integers(0, 256, a.shape)
    for a in (host[1], host[3]):
        a[...] = rng.integers(100, 130, a.shape)
    slots = rng.permutation(65 * 64 + 3).astype(np.int64)                # three of them outside
    say("kv_read %s T=%d" % (out, len(slots)))
    got = cts.kv_read(to_device(host), torch.from_numpy(slots).cuda(), dtype=TORCH[out])
    assert 2 * got[0].numel() * got[0].element_size() >= MB4
    for g, want in zip(got, ob.read(host, slots)):
        assert np.array_equal(f64(g), want)
