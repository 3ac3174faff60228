"""Helpers of the drafted-token GPU tests: trees, their masks, and filled caches."""
import numpy as np
import torch

import paper_2407_00066_amd as cts
from oracle import block as ob

from _block_helpers import ROUND, assert_within, to_device, values
from _gpu_helpers import say

WEIGHTS = {"bf16": 2.0 ** -8, "f32": 2.0 ** -22}


def drafted(rng, n, chain=False):
    """(parents, depths) of n drafts."""
    parents, depth = [], []
    for i in range(n):
        p = i - 1 if chain else (int(rng.integers(max(0, i - 6), i)) if i and rng.random() < 0.85 else -1)
        parents.append(p)
        depth.append(depth[p] + 1 if p >= 0 else 0)
    return parents, depth


def masks(parents, words):
    """uint32 [n, words]: a draft's ancestors and itself."""
    m = np.zeros((len(parents), words), np.uint32)
    for i, p in enumerate(parents):
        if p >= 0:
            m[i] = m[p]
        m[i, i // 32] |= np.uint32(1) << np.uint32(i % 32)
    return m


def filled(rng, pages, page, kvh, d):
    cache = ob.empty_cache(pages, page, kvh, d)
    for a in (cache[0], cache[2]):
        a[...] = rng.integers(0, 256, a.shape)
    for a in (cache[1], cache[3]):
        a[...] = rng.integers(122, 128, a.shape)
    return cache


def make(n_q, n_past, heads, kvh, d, page, dtype="bf16", seed=0, spare=2, big=1.0, words=None, wild=False):
    """A filled cache, a table of pages in no order, queries and trees; wild: masks of no tree, rows that see nothing
    and bits past the drafts among them."""
    rng = np.random.default_rng(seed)
    n_kv = [a + b for a, b in zip(n_q, n_past)]
    need = [-(-max(n, 0) // page) for n in n_kv]
    pages = sum(need) + spare
    order = rng.permutation(pages)
    table, used = np.zeros((len(n_kv), max(need + [1])), np.int32), 0
    for b, n in enumerate(need):
        table[b, :n] = order[used:used + n]
        used += n
    words = words or max(1, -(-max(list(n_q) + [1]) // 32))
    q_start = np.concatenate(([0], np.cumsum(n_q))).astype(np.int32)
    mask, pos = np.zeros((q_start[-1], words), np.uint32), np.zeros(q_start[-1], np.int32)
    for b, (n, past) in enumerate(zip(n_q, n_past)):
        parents, depth = drafted(rng, n)
        at = slice(q_start[b], q_start[b + 1])
        mask[at], pos[at] = masks(parents, words), past + np.array(depth, np.int32)
    if wild:
        mask[...] = rng.integers(0, 2 ** 32, mask.shape, dtype=np.uint32)
        mask[rng.random(len(mask)) < 0.2] = 0
    q64, q = values(rng, (q_start[-1], heads, d), dtype, big)
    return {"cache": filled(rng, pages, page, kvh, d), "table": table, "n_kv": np.array(n_kv, np.int32), "q_start": q_start,
            "q64": q64, "q": q, "heads": heads, "dtype": dtype, "max_q": max(list(n_q) + [1]), "d": d, "mask": mask, "pos": pos}


def i32(a):
    return torch.from_numpy(np.ascontiguousarray(a).view(np.int32)).cuda()


def call(c, window=0, **kw):
    kw.setdefault("max_q", c["max_q"])
    cache = kw.pop("cache", None) or to_device(c["cache"])
    out = cts.kv_tree_attention(kw.pop("q", c["q"]), cache, i32(c["table"]), i32(c["n_kv"]), i32(c["mask"]),
                                q_start=i32(c["q_start"]), window=window, positions=i32(c["pos"]) if window else None, **kw)
    torch.cuda.synchronize()
    return out


def expected(c, window=0, scale=None, max_q=None):
    return ob.tree_attention(c["q64"], c["cache"], c["table"], c["n_kv"], c["q_start"], c["mask"],
                             c["d"] ** -0.5 if scale is None else scale, window, c["pos"], max_q)


def bound(c, want, mag, soft):
    """Half a step of the output; every bf16 weight's rounding (fp32 keeps 24 bits of it, 2^-22 allowed); what fp32 sums leave."""
    return 1.01 * (ROUND[c["dtype"]] * np.abs(want) + WEIGHTS[c["dtype"]] * mag + soft) + 1e-30


def check(c, window=0, scale=None, **kw):
    say("kv_tree_attention %s q=%s kv=%s heads=%d d=%d window=%d" % (c["dtype"], np.diff(c["q_start"]).tolist()[:8],
                                                                     c["n_kv"].tolist()[:8], c["heads"], c["d"], window))
    out = call(c, window, scale=scale, **kw)
    want, mag, soft = expected(c, window, scale, kw.get("max_q"))
    assert_within(out, want, bound(c, want, mag, soft), "kv_tree_attention")
    return out
