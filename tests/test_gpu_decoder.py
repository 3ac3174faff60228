"""The decoder block: every step of it against the oracle, from the values that
the step before left (a rounding may otherwise move a 4-bit code), for prompts,
chunks of prompts and single tokens on one cache."""
import numpy as np
import pytest
import torch

import paper_2407_00066_amd as cts
from oracle import block as ob
from oracle import oracle
from paper_2407_00066_amd import decoder

from _block_helpers import ROUND, assert_within, f64, to_host
from _gpu_helpers import TOL, row_rel_err, say

pytestmark = pytest.mark.gpu

D, HEADS, KV, HD, FF, N, K, R, PAGE = 256, 4, 2, 64, 320, 9, 3, 16, 16


def _bits(t):
    return t.cpu().view(torch.int16).numpy().view(np.uint16)


def _layer(w, x, ids, cluster_of):
    """The oracle's projections of x, side by side as the packed output."""
    W, U, Vt, Sigma = w
    r = U[0].shape[2]
    outs = []
    for m in range(len(W)):
        vt = Vt[:, m * r:(m + 1) * r].contiguous()
        outs.append(oracle.apply(_bits(x), ids, cluster_of, _bits(W[m]), _bits(U[m]), _bits(vt), _bits(Sigma[m])))
    return np.concatenate(outs, axis=1)


def test_block_steps_match_the_oracle(oracle_mod):
    w = decoder.random_weights(D, HEADS, KV, HD, FF, N, K, R, seed=3)
    cos, sin = decoder.rotary_table(200, HD)
    cache = cts.kv_cache(24, PAGE, KV, HD)
    blk = decoder.DecoderBlock(w, HEADS, KV, HD, cache, cos, sin)
    cluster_of = np.arange(N, dtype=np.int32) % K
    dc = torch.from_numpy(cluster_of).cuda()
    tables = [[5, 0, 9, 14], [1, 2, 3, 4], [20, 21, 22, 23]]
    adapter = [7, 0, 4]
    torch.manual_seed(0)
    # a prompt beside a short one; a chunk, a single token and a new prompt; then single tokens
    for who, counts, lens in (([0, 1], [33, 5], [33, 5]), ([0, 1, 2], [20, 1, 40], [53, 6, 40]), ([0, 1, 2], [1, 1, 1], [54, 7, 41])):
        say("decoder block counts=%s lens=%s" % (counts, lens))
        batch = decoder.Batch([adapter[i] for i in who], dc, N, K, counts, lens, [tables[i] for i in who], PAGE)
        ids = np.concatenate([np.full(n, adapter[i], np.int32) for i, n in zip(who, counts)])
        h, y = (torch.randn(batch.T, D, device="cuda").bfloat16() for _ in range(2))
        before = to_host(cache)
        before = tuple(a.copy() for a in before)
        keep = {}
        h2, y2 = blk.forward(h, y, batch, keep)
        torch.cuda.synchronize()
        r = ROUND["bf16"]
        for hin, yin, hk, nk, wn in ((h, y, "h0", "n0", "attn_norm"), (keep["h0"], keep["o"], "h1", "n1", "mlp_norm")):
            rh, rn, mag = ob.block_norm(f64(hin), f64(w[wn]), f64(yin), eps=1e-5)
            assert_within(keep[hk], rh, 1.01 * r * np.abs(rh) + 2.0 ** -22 * mag, hk)
            # (h carries 2^-22 of its terms, at most 16 of its root mean square)
            assert_within(keep[nk], rn, 1.02 * r * np.abs(rn) + 2.0 ** -17 * np.abs(f64(w[wn])) + 1e-30, nk)
        assert row_rel_err(f64(keep["qkv"]), _layer(w["qkv"], keep["n0"], ids, cluster_of)) <= TOL["bf16"]
        qkv = f64(keep["qkv"])
        pos = np.concatenate([np.arange(n - c, n) for c, n in zip(counts, lens)])
        for name, lo, heads in (("q", 0, HEADS), ("k", HEADS, KV)):
            x = qkv[:, lo * HD:(lo + heads) * HD].reshape(-1, heads, HD)
            want, mag = ob.rotary(x, f64(cos), f64(sin), pos[None], [HD // 2])
            assert_within(keep[name], want, 1.01 * r * np.abs(want) + 2.0 ** -22 * mag, name)
        ob.write(before, f64(keep["k"]), f64(keep["v"]), batch.slots.cpu().numpy())
        assert all(np.array_equal(a, b) for a, b in zip(to_host(cache), before))
        start = np.concatenate(([0], np.cumsum(counts)))
        want, mag, soft = ob.attention(f64(keep["q"]), before, batch.table.cpu().numpy(), lens, start, HD ** -0.5)
        assert_within(keep["a"], want, 1.01 * (r * np.abs(want) + 2.0 ** -8 * mag + soft) + 1e-30, "attention")
        assert row_rel_err(f64(keep["o"]), _layer(w["o"], keep["a"].flatten(1), ids, cluster_of)) <= TOL["bf16"]
        assert row_rel_err(f64(keep["gu"]), _layer(w["gate_up"], keep["n1"], ids, cluster_of)) <= TOL["bf16"]
        assert row_rel_err(f64(y2), _layer(w["down"], keep["act"], ids, cluster_of)) <= TOL["bf16"]
        assert torch.equal(h2, keep["h1"]) and torch.equal(y2, keep["y"])


def test_command_runs(capsys):
    say("decoder command")
    decoder.main(["--requests", "3", "--context", "40", "--layers", "1", "--steps", "2"])
    out = capsys.readouterr().out
    assert "prompts: 3 x 40 tokens" in out and "ms a step" in out
