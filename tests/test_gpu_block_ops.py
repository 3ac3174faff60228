"""cts_block_norm and cts_rotary against the oracle.

Norm bounds: outputs are rounded once; a mean of d squares is summed by at most
32 elements a thread and 22 joining steps (64 x 2^-24 of it, half that on its
square root, the root and products a few more); h carries 4 x 2^-24 of its two
terms.  Rotary: one rounding, and 3 x 2^-24 of the products' magnitudes."""
import numpy as np
import pytest
import torch

import paper_2407_00066_amd as cts
from oracle import block as ob

from _block_helpers import ROUND, TORCH, assert_within, f64, values
from _gpu_helpers import say

pytestmark = pytest.mark.gpu
EPS32 = 2.0 ** -24


def _norm_case(T, d, dtype, post, gate, block, seed):
    rng = np.random.default_rng(seed)
    c = {"x": values(rng, (T, d), dtype, 2.0), "weight": values(rng, (d,), dtype)}
    if block:
        c["y"] = values(rng, (T, d), dtype)
        c["post"] = values(rng, (d,), dtype) if post else None
        c["gate"] = values(rng, (T, d) if gate == "token" else (d,), dtype) if gate else None
    return c


def _check_norm(c, h, n, scale, eps, dtype):
    a = [c[k][0] if c.get(k) is not None else None for k in ("x", "weight", "y", "post", "gate")]
    rh, rn, mag = ob.block_norm(a[0], a[1], a[2], a[3], a[4], scale, eps)
    r = ROUND[dtype]
    eh = (64 if c.get("post") is not None else 4) * EPS32 * mag
    assert_within(h, rh, 1.01 * r * np.abs(rh) + eh + 1e-30, "h")
    rs = np.abs(a[1]) / np.sqrt((rh * rh).mean(1, keepdims=True) + eps)
    # an error of h reaches n through its own element, and through the mean by its largest relative share
    share = np.sqrt((eh * eh).mean(1, keepdims=True) / ((rh * rh).mean(1, keepdims=True) + eps))
    assert_within(n, rn, 1.01 * r * np.abs(rn) + rs * eh + (40 * EPS32 + share) * np.abs(rn) + 1e-30, "n")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,d", [(1, 1), (3, 7), (1, 4096), (5, 64), (9, 100), (2, 2048), (7, 2049), (3, 2056), (4, 4104),
                                 (2, 8192), (2, 8200), (1, 16384), (2, 32768), (1, 32767), (301, 520)])
def test_block_norm(T, d, dtype):
    for post, gate, block in ((True, "channel", True), (False, "", True), (False, "token", True), (False, "", False)):
        say("block_norm %s T=%d d=%d post=%d gate=%s block=%d" % (dtype, T, d, post, gate, block))
        c = _norm_case(T, d, dtype, post, gate, block, T + d)
        g = {k: (v[1] if v is not None else None) for k, v in c.items()}
        h, n = cts.block_norm(g["x"], g["weight"], y=g.get("y"), post_weight=g.get("post"), gate=g.get("gate"), scale=0.7,
                              eps=1e-5)
        _check_norm(c, h, n, 0.7, 1e-5, dtype)


@pytest.mark.parametrize("off", [0, 1, 8])
def test_block_norm_strides_and_alignment(off):
    """Rows inside wider ones, at addresses that are and are not multiples of 16 bytes."""
    T, d = 5, 264
    c = _norm_case(T, d, "bf16", True, "token", True, 4)
    wide = {}
    for k in ("x", "y", "gate"):
        wide[k] = torch.full((T, d + 40), 100.0, dtype=torch.bfloat16, device="cuda")[:, off:off + d]
        wide[k].copy_(c[k][1])
    outs = [torch.full((T, d + 24), 7.0, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    h, n = cts.block_norm(wide["x"], c["weight"][1], y=wide["y"], post_weight=c["post"][1], gate=wide["gate"], scale=1.5,
                          eps=1e-6, h_out=outs[0][:, off:off + d], n_out=outs[1][:, off:off + d])
    _check_norm(c, h, n, 1.5, 1e-6, "bf16")
    for o in outs:
        assert bool((o[:, :off] == 7).all()) and bool((o[:, off + d:] == 7).all())


@pytest.mark.parametrize("d", [256, 257, 4096, 9000])
def test_block_norm_in_place(d):
    c = _norm_case(6, d, "bf16", True, "", True, d)
    want = cts.block_norm(c["x"][1], c["weight"][1], y=c["y"][1], post_weight=c["post"][1])
    for over in ("x", "y"):
        t = {k: c[k][1].clone() for k in ("x", "y")}
        h, n = cts.block_norm(t["x"], c["weight"][1], y=t["y"], post_weight=c["post"][1], h_out=t[over],
                              n_out=t["y" if over == "x" else "x"])
        assert torch.equal(h, want[0]) and torch.equal(n, want[1])


def test_block_norm_zero_rows_and_not_finite():
    x = torch.zeros(3, 64, device="cuda")
    w = torch.ones(64, device="cuda")
    h, n = cts.block_norm(x, w, eps=1e-6)
    assert h is x and not n.any()
    x[1, 5] = float("nan")
    n = cts.block_norm(x, w)[1]
    assert torch.isnan(n[1]).all() and not n[[0, 2]].any()
    assert cts.block_norm(x[:0], w)[1].shape == (0, 64)
    big = torch.full((1, 64), 1e18, device="cuda")
    assert torch.allclose(cts.block_norm(big, w)[1], torch.ones(1, 64, device="cuda"))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,heads,kvh,d,rot,sections,inter", [
    (1, 32, 8, 128, 128, None, False), (9, 4, 2, 64, 64, None, True), (13, 3, 1, 256, 128, [20, 20, 24], False),
    (30, 5, 5, 128, 128, [16, 24, 24], True), (7, 2, 1, 64, 16, [1, 7], False), (5, 1, 1, 16, 16, [2, 2, 2, 2], False),
    (257, 6, 2, 128, 64, [0, 32], True)])
def test_rotary(T, heads, kvh, d, rot, sections, inter, dtype):
    say("rotary %s T=%d heads=%d d=%d rot=%d sections=%s" % (dtype, T, heads, d, rot, sections))
    rng = np.random.default_rng(T + d)
    axes = len(sections) if sections else 1
    ang = rng.uniform(0, 100, (50, rot // 2))
    cos, sin = np.cos(ang).astype(np.float32), np.sin(ang).astype(np.float32)
    pos = rng.integers(-2, 53, (axes, T)).astype(np.int32)           # some outside: clamped
    rows64, rows = values(rng, (T, (heads + kvh + 1) * d), dtype)
    q64, k64 = rows64[:, :heads * d].reshape(T, heads, d), rows64[:, heads * d:(heads + kvh) * d].reshape(T, kvh, d)
    q, k = rows[:, :heads * d].unflatten(1, (heads, d)), rows[:, heads * d:(heads + kvh) * d].unflatten(1, (kvh, d))
    dc, ds, dp = torch.from_numpy(cos).cuda(), torch.from_numpy(sin).cuda(), torch.from_numpy(pos).cuda()
    gq, gk = cts.rotary(q, k, dc, ds, dp, sections=sections, interleaved=inter)
    for got, x in ((gq, q64), (gk, k64)):
        want, mag = ob.rotary(x, cos, sin, pos, sections or [rot // 2], inter)
        if rot < d:
            assert np.array_equal(f64(got)[..., rot:], x[..., rot:])
        assert_within(got, want, 1.01 * ROUND[dtype] * np.abs(want) + 3 * EPS32 * mag, "rotary")
    # in place in the packed rows: the rest of the row stays, one side alone works too
    before = rows.clone()
    cts.rotary(q, k, dc, ds, dp, sections=sections, interleaved=inter, q_out=q, k_out=k)
    assert torch.equal(q, gq) and torch.equal(k, gk)
    assert torch.equal(rows[:, (heads + kvh) * d:], before[:, (heads + kvh) * d:])
    only = before[:, heads * d:(heads + kvh) * d].unflatten(1, (kvh, d))
    assert torch.equal(cts.rotary(None, only, dc, ds, dp, sections=sections, interleaved=inter)[1], gk)


def test_rotary_flat_positions_and_no_tokens():
    q = torch.randn(4, 2, 64, device="cuda", dtype=torch.bfloat16)
    ang = torch.rand(9, 32, device="cuda")
    pos = torch.tensor([0, 3, 8, 1], dtype=torch.int32, device="cuda")
    a = cts.rotary(q, None, ang.cos(), ang.sin(), pos)[0]
    assert torch.equal(a, cts.rotary(q, None, ang.cos(), ang.sin(), pos[None])[0])
    assert cts.rotary(q[:0], None, ang.cos(), ang.sin(), pos[:0])[0].shape == (0, 2, 64)
    assert TORCH["f32"] == torch.float32


def test_graph_replays():
    """norm, rotary and a second norm in one graph, replayed with new inputs."""
    x, y = (torch.randn(17, 512, device="cuda").bfloat16() for _ in range(2))
    w = torch.randn(512, device="cuda").bfloat16()
    ang = torch.rand(40, 64, device="cuda")
    cos, sin = ang.cos(), ang.sin()
    pos = torch.arange(17, dtype=torch.int32, device="cuda")
    out = [torch.empty_like(x) for _ in range(3)]

    def step(o):
        cts.block_norm(x, w, y=y, post_weight=w, gate=w, scale=0.5, h_out=o[0], n_out=o[1])
        cts.rotary(o[1].unflatten(1, (4, 128)), None, cos, sin, pos, q_out=o[2].unflatten(1, (4, 128)))
        return o
    step(out)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step(out)
    for _ in range(3):
        x.normal_()
        y.normal_()
        g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, step([torch.empty_like(x) for _ in range(3)])))
