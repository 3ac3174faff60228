"""A decoder block whose every projection carries each token's LoRA: the
multi-adapter layers and the operators around them, as a serving program calls
them.

    python -m paper_2407_00066_amd.decoder [--requests 64] [--context 2000] [--layers 4] [--drafts 8]

runs a prompt, then decode steps, then steps that verify a tree of drafted tokens for each
request, of a small stack on random weights and prints their times: of the layers, and with the
batch's preparation (its lists on the host, their copies, the sort of its tokens).

The residual stream h and the last block's output y travel separately: the
sum h + y is formed by the norm that reads it (block_norm).  Per block:

    h, n = block_norm(h, w_attn, y)         q, k, v = layers(n)       one packed output
    q = kv_append(q, k, v)  in place        positions turned, keys and values into 4-bit pages
    a = kv_attention(q, cache)              o = layer(a)              (drafts: kv_tree_attention)
    h, n = block_norm(h, w_mlp, o)          g, u = layers(n)          one packed output
    y = layer(silu(g) u)
"""
from __future__ import annotations

import argparse
import math
import time

import torch

from . import _binding as cts
from . import block


def draft_tree(parents):
    """(seen, depths) of a sequence's drafts: parents[i] is the draft that draft i follows, an earlier one, or -1 for the
    token before the drafts; seen[i] has a bit for each draft that i follows, and its own."""
    seen, depths = [], []
    for i, p in enumerate(parents):
        if not -1 <= p < i:
            raise ValueError("a draft follows an earlier one, or none (-1)")
        seen.append((seen[p] if p >= 0 else 0) | 1 << i)
        depths.append(depths[p] + 1 if p >= 0 else 0)
    return seen, depths


class Batch:
    """The tokens of one step: each token's LoRA, position and cache slot, and
    each sequence's pages, cached tokens (this step's among them) and query
    rows.  counts (host): tokens of each sequence in this step; kv_len (host):
    cached tokens after it; block_table: lists of pages, one a sequence.
    parents: the tokens are drafts, at most 512 of a sequence; draft_tree's parents for each
    sequence (None: each token follows the one before).  A step holds drafts or other tokens: longer
    parts of prompts go into a batch of their own."""

    def __init__(self, adapter_of, cluster_of, n_adapters, n_clusters, counts, kv_len, block_table, page_size,
                 device="cuda", parents=None):
        def i32(v):
            return torch.tensor(v, dtype=torch.int32, device=device)
        if not counts or not all(0 <= n <= length for n, length in zip(counts, kv_len)):
            raise ValueError("counts must be of one sequence or more, and of no more tokens than kv_len holds with them")
        trees = None
        if parents is not None:
            if len(parents) != len(counts) or any(p is not None and len(p) != n or n > 512 for n, p in zip(counts, parents)):
                raise ValueError("parents must hold one for each of a sequence's tokens, at most 512 (prompts go into a batch of "
                                 "their own)")
            trees = [draft_tree(range(-1, n - 1) if p is None else p) for n, p in zip(counts, parents)]
        ids, pos, slots, start = [], [], [], [0]
        for b, (n, length) in enumerate(zip(counts, kv_len)):
            ids += [adapter_of[b]] * n
            pos += range(length - n, length) if trees is None else [length - n + d for d in trees[b][1]]
            slots += [block_table[b][p // page_size] * page_size + p % page_size for p in range(length - n, length)]
            start.append(start[-1] + n)
        cols = max(len(t) for t in block_table)
        self.T = start[-1]
        self.positions = i32(pos)
        self.slots = torch.tensor(slots, dtype=torch.int64, device=device)
        self.table = i32([list(t) + [0] * (cols - len(t)) for t in block_table])
        self.kv_len, self.q_start = i32(kv_len), i32(start)
        self.max_q, self.max_kv = max(counts), max(kv_len)
        self.mask = None
        if trees is not None:
            words = max(1, -(-self.max_q // 32))
            raw = b"".join(m.to_bytes(4 * words, "little") for seen, _ in trees for m in seen)
            self.mask = torch.frombuffer(bytearray(raw), dtype=torch.int32).view(-1, words).to(device) if raw else \
                torch.empty(0, words, dtype=torch.int32, device=device)
        elif self.max_q == 1 and len(counts) == self.T:
            self.q_start = None                             # one query a sequence
        # the tokens are sorted by cluster and LoRA once for every layer of the step
        self.perm, _, self.bucketing = cts.sort_by_cluster(i32(ids), cluster_of, n_adapters, n_clusters, bucketing=True)


class DecoderBlock:
    """weights: dict with "qkv", "o", "gate_up", "down", each (W, U, Vt, Sigma) as
    apply_multi_packed takes them (lists of W, U and Sigma, the V^T stacked),
    and "attn_norm", "mlp_norm" [d].  cos, sin: the rotary table."""

    def __init__(self, weights, n_heads, n_kv_heads, head_dim, cache: block.KVCache, cos, sin, eps=1e-5):
        self.w, self.cache, self.cos, self.sin, self.eps = weights, cache, cos, sin, eps
        self.n_heads, self.n_kv_heads, self.head_dim = n_heads, n_kv_heads, head_dim

    def _packed(self, x, name, batch):
        return cts.apply_multi_packed(x, *self.w[name], perm=batch.perm, bucketing=batch.bucketing)

    def forward(self, h, y, batch: Batch, keep: dict | None = None):
        """(h, y) after the block; y None for a stack's first.  keep: receives
        the values between the steps."""
        hq, hk, d = self.n_heads, self.n_kv_heads, self.head_dim
        h, n = block.block_norm(h, self.w["attn_norm"], y=y, eps=self.eps)
        qkv = self._packed(n, "qkv", batch)
        if keep is not None:
            keep.update(h0=h, n0=n, qkv=qkv.clone())
        q = qkv[:, :hq * d].unflatten(1, (hq, d))
        k = qkv[:, hq * d:(hq + hk) * d].unflatten(1, (hk, d))
        v = qkv[:, (hq + hk) * d:].unflatten(1, (hk, d))
        block.kv_append(self.cache, q, k, v, batch.slots, self.cos, self.sin, batch.positions, q_out=q,
                        k_out=k if keep is not None else None)
        if batch.mask is not None:
            a = block.kv_tree_attention(q, self.cache, batch.table, batch.kv_len, batch.mask, q_start=batch.q_start,
                                        max_q=max(1, batch.max_q), max_kv=batch.max_kv)
        else:
            a = block.kv_attention(q, self.cache, batch.table, batch.kv_len, q_start=batch.q_start, max_q=batch.max_q,
                                   max_kv=batch.max_kv)
        o = self._packed(a.flatten(1), "o", batch)
        h, n = block.block_norm(h, self.w["mlp_norm"], y=o, eps=self.eps)
        gu = self._packed(n, "gate_up", batch)
        g, u = gu.chunk(2, dim=1)
        act = torch.nn.functional.silu(g) * u
        y = self._packed(act, "down", batch)
        if keep is not None:
            keep.update(q=q, k=k, v=v, a=a, o=o, h1=h, n1=n, gu=gu, act=act, y=y)
        return h, y

    def keep_accepted(self, batch: Batch, path, n_path) -> None:
        """After a step with drafts: draft path[b, i] of sequence b becomes its i-th new token, i < n_path[b] (int32 tensors)."""
        block.kv_keep(self.cache, batch.table, batch.kv_len, batch.q_start, path, n_path)


def rotary_table(n_pos, rot_dim, base=10000.0, device="cuda"):
    half = rot_dim // 2
    angle = torch.arange(n_pos, dtype=torch.float64)[:, None] * base ** (-torch.arange(half, dtype=torch.float64) / half)
    return angle.cos().float().to(device), angle.sin().float().to(device)


def random_weights(d, n_heads, n_kv_heads, head_dim, d_ff, n_adapters, n_clusters, r, seed=0, device="cuda"):
    """Weights of variance 1 / fan-in, adapters of about an eighth of the base's size."""
    g = torch.Generator(device=device)
    g.manual_seed(seed)

    def new(*shape, var):
        return (torch.randn(shape, generator=g, device=device) * math.sqrt(var)).bfloat16()

    def layers(d_in, widths):
        return ([new(w, d_in, var=1 / d_in) for w in widths], [new(n_clusters, w, r, var=1 / w) for w in widths],
                new(n_clusters, len(widths) * r, d_in, var=1 / d_in), [new(n_adapters, r, r, var=1 / r) for _ in widths])
    q, kv = n_heads * head_dim, n_kv_heads * head_dim
    return {"qkv": layers(d, [q, kv, kv]), "o": layers(q, [d]), "gate_up": layers(d, [d_ff, d_ff]),
            "down": layers(d_ff, [d]), "attn_norm": (1 + 0.1 * new(d, var=1)), "mlp_norm": (1 + 0.1 * new(d, var=1))}


def main(argv=None) -> None:
    ap = argparse.ArgumentParser(description="prompt and decode steps of a small stack of decoder blocks")
    ap.add_argument("--requests", type=int, default=64)
    ap.add_argument("--context", type=int, default=2000, help="tokens of a request's prompt")
    ap.add_argument("--layers", type=int, default=4)
    ap.add_argument("--steps", type=int, default=8, help="decode steps, and steps with drafts")
    ap.add_argument("--drafts", type=int, default=8, help="drafted tokens of a request in a step (0: no such steps)")
    a = ap.parse_args(argv)
    if min(a.requests, a.context, a.layers, a.steps) < 1:
        ap.error("requests, context, layers and steps must be at least 1")
    if not 0 <= a.drafts <= 512:
        ap.error("drafts must be from 0 to 512")
    d, heads, kv_heads, head_dim, d_ff, n, K, r, page = 4096, 32, 8, 128, 14336, 100, 4, 64, 16
    total = a.context + a.steps + a.steps * a.drafts
    need = -(-total // page)
    cos, sin = rotary_table(total, head_dim)
    blocks = [DecoderBlock(random_weights(d, heads, kv_heads, head_dim, d_ff, n, K, r, seed=i), heads, kv_heads, head_dim,
                           block.kv_cache(a.requests * need, page, kv_heads, head_dim), cos, sin) for i in range(a.layers)]
    cluster_of = torch.arange(n, dtype=torch.int32, device="cuda") % K
    adapters = [i % n for i in range(a.requests)]
    tables = [range(i * need, (i + 1) * need) for i in range(a.requests)]

    def step(requests, tokens, length, tree=None):
        some = [adapters[i] for i in requests]
        torch.cuda.synchronize()
        t0 = time.perf_counter()
        batch = Batch(some, cluster_of, n, K, [tokens] * len(some), [length] * len(some), [tables[i] for i in requests], page,
                      parents=[tree] * len(some) if tree else None)
        torch.cuda.synchronize()
        prepared = 1e3 * (time.perf_counter() - t0)
        h, y = torch.randn(batch.T, d, device="cuda").bfloat16(), None
        e0, e1 = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        e0.record()
        for b in blocks:
            h, y = b.forward(h, y, batch)
        if tree:                                            # (all layers are done before it is known what is kept)
            for b in blocks:
                b.keep_accepted(batch, path, n_path)
        e1.record()
        e1.synchronize()
        ms = e0.elapsed_time(e1)
        return ms, ms + prepared

    def middle(times):
        return sorted(times)[len(times) // 2]

    chunk = max(1, min(a.requests, 8192 // a.context))
    groups = [range(i, min(i + chunk, a.requests)) for i in range(0, a.requests, chunk)]
    ms = [step(g, a.context, a.context) for g in groups]
    print("prompts: %d x %d tokens, %d layers: %.2f ms, %.2f with the batches' preparation" %
          (a.requests, a.context, a.layers, *map(sum, zip(*ms))))
    ms = [step(range(a.requests), 1, a.context + 1 + i) for i in range(a.steps)]
    print("decode: %d requests, %d layers: %.3f ms a step, %.3f with the batch's preparation" %
          (a.requests, a.layers, *map(middle, zip(*ms))))
    if a.drafts:
        # two tokens follow each, as a drafter's two likeliest do; the model agrees with the last one's branch
        tree = [(i - 1) // 2 for i in range(a.drafts)]
        tree[0], branch = -1, [a.drafts - 1]
        while tree[branch[0]] >= 0:
            branch.insert(0, tree[branch[0]])
        path = torch.tensor([branch] * a.requests, dtype=torch.int32, device="cuda")
        n_path = torch.full((a.requests,), len(branch), dtype=torch.int32, device="cuda")
        ms = [step(range(a.requests), a.drafts, a.context + a.steps + i * len(branch) + a.drafts, tree) for i in range(a.steps)]
        print("drafts: %d requests, %d each, %d layers: %.3f ms a step, %.3f with the batch's preparation" %
              (a.requests, a.drafts, a.layers, *map(middle, zip(*ms))))


if __name__ == "__main__":
    main()
