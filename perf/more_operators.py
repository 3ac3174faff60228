"""Speculative decoding over the 4-bit paged cache, as measurable cases: trees of
drafted tokens are stored, attended to and cut back to what was accepted.

A case is a dict of plain values; "op" names the entry points:
  tree      kv_tree_attention              drafts over their sequence's tokens and, by a mask, each other
  append    kv_append, kv_read             new tokens' positions turned, keys and values stored, the cache read back
  keep      kv_append, kv_keep, kv_read    drafts stored, the accepted ones moved up behind their sequence
With own false, run computes the same in elementary torch operations in 32 bits.

The cache holds blocks of 32 elements along the head dimension: codes of one
sign, two exponent and one mantissa bit (0, 0.5, 1, 1.5, 2, 3, 4, 6) and one
power of two a block, 2^(s - 127) from a byte s.  Keys lie token after token, two codes a byte
(the even element in the low half); values lie in groups of four tokens, so that
eight elements of four tokens are 16 consecutive bytes.

A sequence's n drafts are the last n of its cached tokens.  Bit i of a draft's
mask (32 bits a word, the lowest first) says that it sees draft i; all see the
tokens before the drafts.
"""
import math
import random

import torch

own = False

BF16, F32, F64 = torch.bfloat16, torch.float32, torch.float64
DTYPES = {"bf16": BF16, "f32": F32}
BLOCK = 32


# ---------------------------------------------------------------- cases
def _tree(name, n_q, n_past, heads, kv_heads, d, page, window=0, dtype="bf16"):
    """n_q, n_past: drafts of a sequence and cached tokens before them, as text."""
    return {"name": name, "op": "tree", "n_q": n_q, "n_past": n_past, "heads": heads, "kv_heads": kv_heads, "d": d,
            "page": page, "window": window, "dtype": dtype}


def _append(name, T, slots, heads, kv_heads, d, page, rot=128, axes=1, interleaved=False, n_pos=8192, dtype="bf16"):
    return {"name": name, "op": "append", "T": T, "slots": slots, "heads": heads, "kv_heads": kv_heads, "d": d, "page": page,
            "rot": rot, "axes": axes, "interleaved": interleaved, "n_pos": n_pos, "dtype": dtype}


def _keep(name, n_q, n_past, kv_heads, d, page, dtype="bf16"):
    return {"name": name, "op": "keep", "n_q": n_q, "n_past": n_past, "kv_heads": kv_heads, "d": d, "page": page,
            "rot": d, "n_pos": 8192, "dtype": dtype}


def _lens(seed, n, lo, hi):
    rng = random.Random(seed)
    return " ".join(str(rng.randint(lo, hi)) for _ in range(n))


def listed():
    return [
        # one request answering alone, seven tokens drafted for it
        _tree("tree_1", "7", "702", 32, 8, 128, 16),
        # 64 requests of mixed age with small trees
        _tree("tree_64", _lens(21, 64, 3, 16), _lens(22, 64, 40, 4000), 32, 8, 128, 16),
        # many requests with a few drafts each
        _tree("tree_200", _lens(23, 200, 1, 6), _lens(24, 200, 30, 2000), 32, 8, 128, 16),
        # a few requests with wide trees
        _tree("tree_wide", _lens(25, 8, 40, 64), _lens(26, 8, 300, 8000), 32, 8, 128, 32),
        # wide trees behind long documents
        _tree("tree_long", "64 31 50", "65472 39970 131022", 32, 8, 128, 64),
        # 32-bit queries and a sliding window; drafts of an empty sequence and a padded row among them
        _tree("tree_f32", "5 1 12 7 33 5 16 2", "1495 32 0 805 2014 0 584 4097", 16, 4, 64, 32, 1024, "f32"),
        # large heads, all queries of one key/value head
        _tree("tree_d256", _lens(27, 12, 9, 20), _lens(28, 12, 200, 6000), 8, 1, 256, 64),
        # a decode step's new tokens, from the packed q/k/v rows
        _append("append_33", 33, 64, 32, 8, 128, 16),
        # prompts being stored
        _append("append_prefill", 8191, 8704, 32, 8, 128, 16),
        # 32-bit rows, positions in time, height and width over half of each head
        _append("append_axes_f32", 2003, 2560, 20, 4, 128, 64, rot=64, axes=3, dtype="f32"),
        # one request's verified drafts
        _keep("keep_1", "7", "50", 8, 128, 16),
        # a batch's
        _keep("keep_64", _lens(29, 64, 1, 33), _lens(30, 64, 0, 200), 8, 128, 16),
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _draw_heads(rng):
    kv = rng.choice((1, 2, 4, 8))
    return kv * rng.choice((1, 2, 3, 4, 4, 5, 7, 8, 8)), kv


def _text(v):
    return " ".join(map(str, v))


def _draw_tree(rng):
    heads, kv_heads = _draw_heads(rng)
    d, page = rng.choice((64, 128, 128, 128, 256)), rng.choice((16, 16, 32, 64, 128))
    dtype = "f32" if rng.random() < 0.2 else "bf16"
    window = _log_int(rng, 16, 4096) if rng.random() < 0.25 else 0
    B = _log_int(rng, 1, 200)
    drafts, context = _log_int(rng, 1, 200), _log_int(rng, 8, 131072)
    tokens = 2.3e5 * 8 * 128 / (kv_heads * d)
    products = (4.8e10 if dtype == "bf16" else 4e9) / (heads * d)
    n_q, n_past = [], []
    for _ in range(B):
        n = rng.randint(max(1, drafts // 4), drafts)
        past = 0 if rng.random() < 0.03 else rng.randint(context // 8, context)
        past = int(min(past, max(0, tokens), max(0, products / n - n)))
        tokens -= past + n
        products -= n * (past + n)
        if n_q and (tokens < 0 or products < 0):
            break
        n_q.append(n)
        n_past.append(past)
    c = _tree("", _text(n_q), _text(n_past), heads, kv_heads, d, page, window, dtype)
    del c["name"]
    return c


def draw(rng):
    pick = rng.random()
    if pick < 0.55:
        return _draw_tree(rng)
    heads, kv_heads = _draw_heads(rng)
    d, page = rng.choice((64, 128, 128, 256)), rng.choice((16, 32, 64, 128))
    dtype = "f32" if rng.random() < 0.25 else "bf16"
    if pick < 0.83:
        T = min(_log_int(rng, 1, 8191), 8191 * 40 * 128 // ((heads + kv_heads) * d))
        slots = (T * rng.randint(10, 12) // 10 + page) // page * page
        c = _append("", T, slots, heads, kv_heads, d, page, rng.choice((d, d, d // 2)), rng.choice((1, 1, 2, 3)),
                    rng.random() < 0.3, _log_int(rng, 256, 65536), dtype)
    else:
        B, most = _log_int(rng, 1, 100), _log_int(rng, 1, 64)
        n_q = [rng.randint(1, most) for _ in range(B)]
        c = _keep("", _text(n_q), _text(rng.randint(0, 150) for _ in n_q), kv_heads, d, page, dtype)
    del c["name"]
    return c


def _ints(text):
    return [int(v) for v in text.split()]


def _sections(c):
    """Frequencies of each axis: near-equal shares, the first ones larger."""
    half, a = c["rot"] // 2, c.get("axes", 1)
    return [half // a + (1 if i < half % a else 0) for i in range(a)]


# ---------------------------------------------------------------- the cache in torch operations
E2M1 = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def _quantize(x):
    """(codes, scale bytes) of x [..., d]: uint8 [..., d] and [..., d / 32]."""
    x = x.float().unflatten(-1, (-1, BLOCK))
    top = x.abs().amax(-1)
    s = ((top.view(torch.int32) + (1 << 21)) >> 23) - 2       # the largest rounds to 6 at most
    s = torch.where(torch.isfinite(top), s.clamp(1, 252), 255)
    y = x / (s.clamp_max(254) << 23).view(F32).unsqueeze(-1)
    m = y.abs().unsqueeze(-1)
    over = torch.tensor((0.25, 1.25, 2.5, 5.0), device=x.device)          # ties go to the even code
    reach = torch.tensor((0.75, 1.75, 3.5), device=x.device)
    code = ((m > over).sum(-1) + (m >= reach).sum(-1)).to(torch.uint8)
    code = code + (torch.signbit(y).to(torch.uint8) << 3)
    code = torch.where(torch.isfinite(top).unsqueeze(-1), code, torch.zeros_like(code))
    return code.flatten(-2), s.to(torch.uint8)


def _pack(code):
    return code[..., 0::2] | (code[..., 1::2] << 4)


def _pairs(device):
    """Both values of every byte, [256, 2]."""
    v = torch.tensor(E2M1 + tuple(-e for e in E2M1), device=device)
    b = torch.arange(256, device=device)
    return torch.stack((v[b & 15], v[b >> 4]), 1)


def _scale(s):
    f = (s.int().clamp_min(1) << 23).view(F32)
    return torch.where(s == 255, torch.full_like(f, float("nan")), f)


def _values(codes, scales):
    """Values [..., d] of packed codes [..., d / 2] and scale bytes [..., d / 32]."""
    v = torch.index_select(_pairs(codes.device), 0, codes.reshape(-1).int()).view(*codes.shape[:-1], -1)
    return (v.unflatten(-1, (-1, BLOCK)) * _scale(scales).unsqueeze(-1)).flatten(-2)


def _v_values(codes, scales):
    """[..., page, d] from codes [..., page / 4, d / 8, 4, 4] and scales [..., page / 4, d / 32, 4]."""
    return _values(codes.transpose(-3, -2).flatten(-2).flatten(-3, -2), scales.transpose(-2, -1).flatten(-3, -2))


def _bytes_at(cache, slots):
    """The slots' bytes in each of the cache's four arrays."""
    kc, ks, vc, vs = cache
    page = kc.shape[2]
    p, o = slots // page, slots % page
    return kc[p, :, o], ks[p, :, o], vc[p, :, o // 4, :, o % 4], vs[p, :, o // 4, :, o % 4]


def _put_bytes(cache, slots, new):
    kc, ks, vc, vs = cache
    page = kc.shape[2]
    p, o = slots // page, slots % page
    kc[p, :, o], ks[p, :, o], vc[p, :, o // 4, :, o % 4], vs[p, :, o // 4, :, o % 4] = new


def _store(cache, k, v, slots):
    """New tokens into the cache's four arrays."""
    (kc, ks), (vc, vs) = _quantize(k), _quantize(v)
    _put_bytes(cache, slots, (_pack(kc), ks, _pack(vc).unflatten(-1, (-1, 4)), vs))


def _load(cache, slots):
    kc, ks, vc, vs = _bytes_at(cache, slots)
    return _values(kc, ks), _values(vc.flatten(-2), vs)


def _empty_cache(pages, page, heads, d, device="cuda"):
    new = lambda *shape: torch.zeros(shape, dtype=torch.uint8, device=device)
    return (new(pages, heads, page, d // 2), new(pages, heads, page, d // BLOCK),
            new(pages, heads, page // 4, d // 8, 4, 4), new(pages, heads, page // 4, d // BLOCK, 4))


# ---------------------------------------------------------------- inputs
class _Draw:
    def __init__(self, seed, dtype):
        self.g = torch.Generator(device="cuda")
        self.g.manual_seed(seed)
        self.dtype = dtype

    def __call__(self, shape, std=1.0):
        return torch.randn(shape, generator=self.g, device="cuda").mul_(std).to(self.dtype)


def _i32(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def _keys(dr, T, heads, d):
    """Keys with a few channels far larger than the rest, as trained models have."""
    std = torch.ones(heads, d, device="cuda")
    std[:, ::29] = 4.0
    return (dr((T, heads, d)).float() * std).to(dr.dtype)


def _filled_cache(dr, pages, page, H, d):
    cache = _empty_cache(pages, page, H, d)
    part = max(1, 65536 // page)
    for at in range(0, pages, part):
        slots = torch.arange(at * page, min(pages, at + part) * page, device="cuda")
        _store(cache, _keys(dr, len(slots), H, d), dr((len(slots), H, d)), slots)
    return cache


def _tables(n_kv, page, seed):
    """Pages taken in no order: lists of one length, and how many pages there are."""
    need = [(n + page - 1) // page for n in n_kv]
    order = list(range(sum(need) + 3))
    random.Random(seed * 7 + 3).shuffle(order)
    table, used = [], 0
    for n in need:
        table.append(order[used:used + n] + [0] * (max(need) - n))
        used += n
    return table, len(order)


def _drafted(n, rng):
    """(parents, depths) of n drafts: a draft follows one of the dozen before it, or starts a branch."""
    parents, depth = [], []
    for i in range(n):
        p = rng.randint(max(0, i - 12), i - 1) if i and rng.random() < 0.9 else -1
        parents.append(p)
        depth.append(depth[p] + 1 if p >= 0 else 0)
    return parents, depth


def _tree_inputs(c, seed):
    dr, rng = _Draw(seed, DTYPES[c["dtype"]]), random.Random(seed * 7 + 6)
    n_q, n_past, page, d, H = _ints(c["n_q"]), _ints(c["n_past"]), c["page"], c["d"], c["kv_heads"]
    n_kv = [a + b for a, b in zip(n_q, n_past)]
    table, pages = _tables(n_kv, page, seed)
    words = (max(n_q) + 31) // 32
    start, masks, positions = [0], [], []
    for n, past in zip(n_q, n_past):
        parents, depth = _drafted(n, rng)
        seen = []
        for i, p in enumerate(parents):
            seen.append((seen[p] if p >= 0 else 0) | 1 << i)
        if n > 4 and rng.random() < 0.1:                # the last draft is padding: it sees none, itself neither
            seen[-1] = 0
        for m, dep in zip(seen, depth):
            w = [m >> (32 * j) & 0xffffffff for j in range(words)]
            masks.append([x - (1 << 32) if x >> 31 else x for x in w])
            positions.append(past + dep)
        start.append(start[-1] + n)
    cache = _filled_cache(dr, pages, page, H, d)
    # queries are a part of the packed q/k/v rows
    rows = dr((start[-1], (c["heads"] + 2 * H) * d))
    return {"cache": cache, "q": rows[:, :c["heads"] * d].unflatten(1, (c["heads"], d)), "table": _i32(table),
            "kv_len": _i32(n_kv), "q_start": _i32(start), "mask": _i32(masks), "positions": _i32(positions)}


def _rotary_table(c):
    half = c["rot"] // 2
    freq = 10000.0 ** (-torch.arange(half, dtype=F64) / half)
    angle = torch.arange(c["n_pos"], dtype=F64)[:, None] * freq
    return angle.cos().float().cuda(), angle.sin().float().cuda()


def _packed_rows(dr, T, heads, H, d):
    """(q, k, v), parts of packed rows."""
    rows = dr((T, (heads + 2 * H) * d))
    rows[:, heads * d:(heads + H) * d] = _keys(dr, T, H, d).flatten(1)
    rows = rows.unflatten(1, (heads + 2 * H, d))
    return rows[:, :heads], rows[:, heads:heads + H], rows[:, heads + H:]


def _append_inputs(c, seed):
    dr = _Draw(seed, DTYPES[c["dtype"]])
    T, H, d, n, page = c["T"], c["kv_heads"], c["d"], c["slots"], c["page"]
    order = list(range(n // page))
    random.Random(seed * 7 + 4).shuffle(order)          # prompts take whole pages, in no order
    flat = [p * page + o for p in order for o in range(page)]
    if T < 256:                                         # decode: one token here and there
        flat = random.Random(seed * 7 + 5).sample(flat, T)
    q, k, v = _packed_rows(dr, T, c["heads"], H, d)
    cos, sin = _rotary_table(c)
    pos = torch.randint(0, c["n_pos"], (c["axes"], T), generator=dr.g, device="cuda", dtype=torch.int32)
    return {"cache": _filled_cache(dr, n // page, page, H, d), "slots": torch.tensor(flat[:T], device="cuda"),
            "every": torch.arange(n, device="cuda"), "q": q, "k": k, "v": v, "cos": cos, "sin": sin, "pos": pos}


def _keep_inputs(c, seed):
    dr, rng = _Draw(seed, DTYPES[c["dtype"]]), random.Random(seed * 7 + 6)
    n_q, n_past, page, d, H = _ints(c["n_q"]), _ints(c["n_past"]), c["page"], c["d"], c["kv_heads"]
    n_kv = [a + b for a, b in zip(n_q, n_past)]
    table, pages = _tables(n_kv, page, seed)
    start, pos, slots, paths = [0], [], [], []
    for b, (n, past) in enumerate(zip(n_q, n_past)):
        parents, depth = _drafted(n, rng)
        leaf, path = rng.randrange(n), []
        while leaf >= 0:                                # what the model agreed with: from a draft back to its branch's start
            path.insert(0, leaf)
            leaf = parents[leaf]
        paths.append(path if rng.random() < 0.9 else [])
        pos += [past + dep for dep in depth]
        slots += [table[b][t // page] * page + t % page for t in range(past, past + n)]
        start.append(start[-1] + n)
    most = max(max(map(len, paths)), 1)
    _, k, v = _packed_rows(dr, start[-1], 4 * H, H, d)
    cos, sin = _rotary_table(c)
    return {"cache": _filled_cache(dr, pages, page, H, d), "slots": torch.tensor(slots, device="cuda"),
            "every": torch.arange(pages * page, device="cuda"), "q": None, "k": k, "v": v, "cos": cos, "sin": sin,
            "pos": _i32([pos]), "table": _i32(table), "kv_len": _i32(n_kv), "q_start": _i32(start),
            "path": _i32([p + [-1] * (most - len(p)) for p in paths]), "n_path": _i32([len(p) for p in paths])}


_INPUTS = {"tree": _tree_inputs, "append": _append_inputs, "keep": _keep_inputs}


def prepare(case, seed):
    s = _INPUTS[case["op"]](case, seed)
    s["case"] = case
    if case["op"] == "tree":
        # a serving program knows its batch's lengths on the host as well
        s["n_q"] = _ints(case["n_q"])
        s["n_kv"] = [a + b for a, b in zip(s["n_q"], _ints(case["n_past"]))]
    if own:
        import paper_2407_00066_amd as cts
        s["kv"] = cts.KVCache(*s["cache"])
        if case["op"] == "tree":
            need = cts.kv_tree_attention_workspace_size(s["q"], s["kv"], len(s["n_q"]), max(s["n_q"]), max(s["n_kv"]),
                                                        window=case["window"])
            s["ws"] = torch.empty(need, dtype=torch.uint8, device="cuda")
    return s


# ---------------------------------------------------------------- one pass
def run(s):
    return _run_own(s) if own else _PLAIN[s["case"]["op"]](s)


def _run_own(s):
    import paper_2407_00066_amd as cts
    c = s["case"]
    if c["op"] == "tree":
        return cts.kv_tree_attention(s["q"], s["kv"], s["table"], s["kv_len"], s["mask"], q_start=s["q_start"],
                                     max_q=max(s["n_q"]), max_kv=max(s["n_kv"]), window=c["window"],
                                     positions=s["positions"] if c["window"] else None, workspace=s["ws"])
    q = cts.kv_append(s["kv"], s["q"], s["k"], s["v"], s["slots"], s["cos"], s["sin"], s["pos"], sections=_sections(c),
                      interleaved=c.get("interleaved", False))
    if c["op"] == "append":
        return (q, *cts.kv_read(s["kv"], s["every"], dtype=DTYPES[c["dtype"]]))
    cts.kv_keep(s["kv"], s["table"], s["kv_len"], s["q_start"], s["path"], s["n_path"])
    return cts.kv_read(s["kv"], s["every"], dtype=DTYPES[c["dtype"]])


def _plain_group(s, rows, out):
    """Some sequences, padded to the longest of them and to the most drafts."""
    c, q = s["case"], s["q"]
    kc, ks, vc, vs = s["cache"]
    H, d, page = c["kv_heads"], c["d"], c["page"]
    G, N, L = c["heads"] // H, max(s["n_q"][r] for r in rows), max(s["n_kv"][r] for r in rows)
    at = torch.tensor(rows, device="cuda")
    pages = s["table"][at, :(L + page - 1) // page]
    k, v = _values(kc[pages], ks[pages]), _v_values(vc[pages], vs[pages])      # [b, pages, H, page, d]
    k, v = k.transpose(1, 2).flatten(2, 3)[:, :, :L], v.transpose(1, 2).flatten(2, 3)[:, :, :L]
    start, n = s["q_start"][at].long()[:, None], (s["q_start"][at + 1] - s["q_start"][at])[:, None]
    j = torch.arange(N, device="cuda")
    real = j < n                                                               # [b, N]: rows that are there
    row = (start + j).clamp_max(len(q) - 1)
    qq = q[row].float().unflatten(2, (H, G)).permute(0, 2, 1, 3, 4).flatten(2, 3)      # [b, H, N G, d]
    score = torch.matmul(qq, k.transpose(-1, -2)) / math.sqrt(d)
    t = torch.arange(L, device="cuda")
    past = s["kv_len"][at][:, None] - n
    draft = t - past                                                           # [b, L]
    bits = (s["mask"][row].unsqueeze(-1) >> torch.arange(32, device="cuda") & 1).flatten(2).bool()     # [b, N, 32 words]
    in_tree = torch.gather(bits, 2, draft.clamp(0, bits.shape[2] - 1)[:, None].expand(-1, N, -1))
    seen = torch.where((draft < 0)[:, None], torch.ones_like(in_tree), in_tree & (draft < n)[:, None])
    if c["window"]:
        seen &= (draft >= 0)[:, None] | (t > s["positions"][row][..., None] - c["window"])
    seen = seen[:, None, :, None, :].expand(-1, 1, N, G, L).flatten(2, 3)
    score = score.masked_fill(~seen, float("-inf"))
    top = score.amax(-1, keepdim=True).clamp_min(-3e38)
    p = torch.exp(score - top)
    o = torch.matmul(p, v) / p.sum(-1, keepdim=True).clamp_min(1e-30)
    o = o.unflatten(2, (N, G)).permute(0, 2, 1, 3, 4).flatten(2, 3).to(q.dtype)        # [b, N, heads, d]
    out[row[real]] = o[real]


def _plain_tree(s):
    c = s["case"]
    out = torch.empty(s["q"].shape, dtype=s["q"].dtype, device="cuda")
    left = sorted(range(len(s["n_q"])), key=lambda r: s["n_kv"][r])
    while left:                                         # padded scores and tokens of a gigabyte or so at a time
        L, N = s["n_kv"][left[-1]], max(s["n_q"])
        take = max(1, min(2 ** 28 // (L * c["heads"] * N), 2 ** 28 // (L * c["kv_heads"] * c["d"])))
        _plain_group(s, left[-take:], out)
        del left[-take:]
    return out


def _turned(x, s):
    """x at its positions.  The sine's product is rounded to 32 bits, the cosine's is not (a fused
    multiply-add): a key may lie next to the border of two codes."""
    c = s["case"]
    n, half = torch.tensor(_sections(c), device="cuda"), c["rot"] // 2
    axis = torch.repeat_interleave(torch.arange(len(n), device="cuda"), n, output_size=half)
    at = s["pos"][axis].long().t()                                             # [T, half]
    pair = torch.arange(half, device="cuda")
    cos, sin = s["cos"][at, pair][:, None], s["sin"][at, pair][:, None]
    o = x.float().clone()
    lo, hi = (o[..., 0:c["rot"]:2], o[..., 1:c["rot"]:2]) if c.get("interleaved") else (o[..., :half], o[..., half:c["rot"]])
    new_lo = (lo.double() * cos.double() - (hi * sin).double()).float()
    new_hi = (hi.double() * cos.double() + (lo * sin).double()).float()
    lo.copy_(new_lo)
    hi.copy_(new_hi)
    return o.to(x.dtype)


def _plain_append(s):
    q = _turned(s["q"], s)
    _store(s["cache"], _turned(s["k"], s), s["v"], s["slots"])
    k, v = _load(s["cache"], s["every"])
    return q, k.to(q.dtype), v.to(q.dtype)


def _moves(s):
    """(from, to): the slots that the accepted drafts leave and take."""
    page, path = s["case"]["page"], s["path"].long()
    i = torch.arange(path.shape[1], device="cuda")
    past = (s["kv_len"] - (s["q_start"][1:] - s["q_start"][:-1])).long()[:, None]
    real = i < s["n_path"][:, None]
    slot = lambda t: (torch.gather(s["table"].long(), 1, t // page) * page + t % page)[real]
    return slot(past + path.clamp_min(0)), slot((past + i).clamp_max(s["table"].shape[1] * page - 1))


def _plain_keep(s):
    dt = s["k"].dtype
    _store(s["cache"], _turned(s["k"], s), s["v"], s["slots"])
    left, taken = _moves(s)
    _put_bytes(s["cache"], taken, _bytes_at(s["cache"], left))
    k, v = _load(s["cache"], s["every"])
    return k.to(dt), v.to(dt)


_PLAIN = {"tree": _plain_tree, "append": _plain_append, "keep": _plain_keep}


# ---------------------------------------------------------------- work
def work(case):
    c = case
    e = 2.0 if c["dtype"] == "bf16" else 4.0
    row = 2.0 * c["kv_heads"] * c["d"]                                         # elements of a token's keys and values
    packed = row * (0.5 + 1.0 / BLOCK)
    if c["op"] == "tree":
        n_q, n_past = _ints(c["n_q"]), _ints(c["n_past"])
        past = [min(p, c["window"]) if c["window"] else p for p in n_past]     # (that a draft without others before it sees)
        tokens = sum(n_q) + sum(past)
        pages = sum((n + t + c["page"] - 1) // c["page"] for n, t in zip(n_q, past))
        words = (max(n_q) + 31) // 32
        return {"bytes": 2 * e * sum(n_q) * c["heads"] * c["d"] + packed * tokens + 4.0 * (pages + 2 * len(n_q) + sum(n_q) * words),
                "flops": 4.0 * c["d"] * c["heads"] * sum(n * (t + 1) for n, t in zip(n_q, past))}
    turn = 4.0 * (c["rot"] + c.get("axes", 1)) + 8                             # angles, positions and the slot
    if c["op"] == "append":
        T, wide = c["T"], c["heads"] * c["d"]
        # queries read and written, keys and values read and stored, then every slot read (a new token's straight from its store)
        return {"bytes": T * (2 * e * wide + e * row + packed + turn) + (c["slots"] - T) * packed + c["slots"] * (e * row + 8),
                "flops": 3.0 * T * (c["heads"] + c["kv_heads"]) * c["rot"] + (3.0 * T + c["slots"]) * row}
    n_q, n_past = _ints(c["n_q"]), _ints(c["n_past"])
    T = sum(n_q)
    slots = (sum((n + p + c["page"] - 1) // c["page"] for n, p in zip(n_q, n_past)) + 3.0) * c["page"]
    return {"bytes": T * (e * row + packed + turn) + (slots - T) * packed + slots * (e * row + 8),
            "flops": 3.0 * T * c["kv_heads"] * c["rot"] + (3.0 * T + slots) * row}


# ---------------------------------------------------------------- 64-bit results
def _exact_values(code, scale):
    """float64 from one code an element (any shape) and a scale byte an element."""
    c = code.long()
    e, m = (c >> 1) & 3, (c & 1).double()
    mag = torch.where(e == 0, 0.5 * m, (1 + 0.5 * m) * torch.exp2((e - 1).double()))
    return torch.where(c >= 8, -mag, mag) * torch.exp2(scale.double() - 127)


def _exact_rows(cache, p, o):
    """Keys and values [n, H, d] of the slots (page p, offset o)."""
    outs = []
    for which in (0, 2):
        codes, scales = cache[which], cache[which + 1]
        if which == 0:
            by, sc = codes[p, :, o], scales[p, :, o]
        else:
            n = torch.arange(len(p), device="cuda")
            by, sc = codes[p, :, o >> 2][n, :, :, o & 3].flatten(2), scales[p, :, o >> 2][n, :, :, o & 3]
        code = torch.stack((by & 15, by >> 4), -1).flatten(2)
        outs.append(_exact_values(code, sc.repeat_interleave(BLOCK, 2)))
    return outs


def _exact_tree(c, s):
    out = torch.zeros(s["q"].shape, dtype=F64, device="cuda")
    G, at = c["heads"] // c["kv_heads"], 0
    words = s["mask"].cpu().tolist()
    where = s["positions"].cpu().tolist()
    for b, (n, past) in enumerate(zip(_ints(c["n_q"]), _ints(c["n_past"]))):
        t = torch.arange(past + n, device="cuda")
        K, V = [], []
        for lo in range(0, past + n, 32768):
            part = t[lo:lo + 32768]
            k, v = _exact_rows(s["cache"], s["table"][b].long()[part // c["page"]], part % c["page"])
            K.append(k)
            V.append(v)
        K, V = torch.cat(K), torch.cat(V)
        hidden = []
        for j in range(at, at + n):
            first = max(0, where[j] - c["window"] + 1) if c["window"] else 0
            hidden.append([words[j][i // 32] >> (i % 32) & 1 == 0 for i in range(n)] + [first])
        tree = torch.tensor([h[:n] for h in hidden], device="cuda").view(n, n)
        first = torch.tensor([h[n] for h in hidden], device="cuda")
        hidden = torch.cat((t[None, :past] < first[:, None], tree), 1)
        for h in range(c["heads"]):
            x = (s["q"][at:at + n, h].double() @ K[:, h // G].t()) * c["d"] ** -0.5
            x[hidden] = -math.inf
            w = torch.softmax(x, 1)
            w[hidden.all(1)] = 0                        # a row that sees nothing
            out[at:at + n, h] = w @ V[:, h // G]
        at += n
    return out


def _exact_round(x):
    """The stored values of x: nearest multiples of a power of two per block, found from the block's largest."""
    x = x.double().unflatten(-1, (-1, BLOCK))
    top = x.abs().amax(-1, keepdim=True)
    f, e = torch.frexp(top)                                                  # top = f 2^e, f in [0.5, 1)
    e = torch.where(f >= 0.875, e - 2, e - 3)
    e = torch.where(top == 0, torch.full_like(e, -126), e).clamp_min(-126)
    unit = torch.exp2(e.double())
    m = x.abs() / unit
    step = torch.where(m < 2, 0.5, torch.where(m < 4, 1.0, 2.0))
    return (torch.sign(x) * torch.round(m / step) * step * unit).flatten(-2)


def _exact_turned(c, s, x):
    axis = [a for a, n in enumerate(_sections(c)) for _ in range(n)]
    o = x.double()
    for j, a in enumerate(axis):
        at = s["pos"][a].long()
        co, si = s["cos"][at, j].double()[:, None], s["sin"][at, j].double()[:, None]
        i0, i1 = (2 * j, 2 * j + 1) if c.get("interleaved") else (j, j + c["rot"] // 2)
        a0, a1 = o[:, :, i0].clone(), o[:, :, i1].clone()
        o[:, :, i0], o[:, :, i1] = a0 * co - a1 * si, a1 * co + a0 * si
    return o


def _exact_stored(c, s):
    """Every slot's keys and values once the new tokens are in: turned keys are rounded to their type, then stored."""
    k, v = _exact_rows(s["cache"], s["every"] // c["page"], s["every"] % c["page"])
    k[s["slots"]] = _exact_round(_exact_turned(c, s, s["k"]).to(s["k"].dtype))
    v[s["slots"]] = _exact_round(s["v"])
    return k, v


def _exact_append(c, s):
    return (_exact_turned(c, s, s["q"]), *_exact_stored(c, s))


def _exact_keep(c, s):
    k, v = _exact_stored(c, s)
    old_k, old_v = k.clone(), v.clone()
    table, paths, lens = s["table"].cpu().tolist(), s["path"].cpu().tolist(), s["n_path"].cpu().tolist()
    for b, past in enumerate(_ints(c["n_past"])):
        slot = lambda t: table[b][t // c["page"]] * c["page"] + t % c["page"]
        left = [slot(past + i) for i in paths[b][:lens[b]]]
        taken = [slot(past + i) for i in range(lens[b])]
        k[taken], v[taken] = old_k[left], old_v[left]
    return k, v


def exact(case, seed):
    s = _INPUTS[case["op"]](case, seed)
    return {"tree": _exact_tree, "append": _exact_append, "keep": _exact_keep}[case["op"]](case, s)
