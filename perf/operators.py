"""Cases for timing the operators of a speculative decoding step on one GPU: norm and rotation of queries and keys,
the paged key-value cache in 8 bits, attention of drafted tokens over it.

listed() and draw() give cases, prepare() makes what a serving program has in hand before the call, run() makes
one pass and work() states what a pass cannot do without.  exact() computes the results in 64 bits from the
definitions.  With `own` false, run() is the plain form of the operators in elementary operations in 32 bits;
with `own` true it calls paper_2602_06072_amd.binding.

The lengths of a case come from its own "structure" number, so that work() knows them; values come from the seed.

op      one pass is
rope    qk_norm_rope: norm and rotation of the queries and keys of a layer
cache   kv_cache_write of new tokens, then kv_cache_read of all tokens of the requests, as before the attention
        of a prompt in chunks
tree    tree_attn: attention of the drafted tokens of every request (one token: a plain decode step)
step    qkv_cache_write, tree_attn, kv_cache_keep: norm, rotation and cache write of the drafted tokens of a
        layer, their attention, and the accepted ones moved up behind the context

The cache (types "f8" and "bf16"): K [blocks][Hkv][page][d]; V [blocks][Hkv][page / 4][d][4], four tokens
interleaved; with "f8" E4M3 codes and scales [blocks][Hkv][2][page] (K, V), powers of two, one for each token and
head: 2^E with the smallest E that keeps the row's largest finite magnitude within 448, at least -126.
"""
import math

import numpy as np
import torch

own = False
DEV = "cuda"
EPS = 1e-6
F8_MAX = 448.0


# ---------------------------------------------------------------------------------------------
# cases
# ---------------------------------------------------------------------------------------------

def _rope(name, tokens, heads, rot, axes=1, interleaved=False, norm=True, dtype="bf16", out="bf16", structure=0):
    """tokens rows; rot of the d columns rotated, positions of `axes` axes."""
    Hq, Hkv, d = heads
    return dict(name=name, op="rope", tokens=tokens, Hq=Hq, Hkv=Hkv, d=d, rot=rot, axes=axes, interleaved=interleaved,
                norm=norm, dtype=dtype, out=out, structure=structure)


def _cache(name, n, ctx_lo, ctx_hi, new_lo, new_hi, heads, cache="f8", dtype="bf16", out="bf16", page=16, structure=0):
    """n requests with a context in [ctx_lo, ctx_hi], new tokens behind it in [new_lo, new_hi]."""
    Hkv, d = heads
    return dict(name=name, op="cache", n=n, ctx_lo=ctx_lo, ctx_hi=ctx_hi, skew=1, new_lo=new_lo, new_hi=new_hi, Hkv=Hkv,
                d=d, cache=cache, dtype=dtype, out=out, page=page, structure=structure)


def _tree(name, op, n, ctx_lo, ctx_hi, new_lo, new_hi, heads, cache="f8", chain=False, skew=1, page=16, structure=0):
    """n requests; context in [ctx_lo, ctx_hi] (skew 1: uniform, 3: mostly short), drafted tokens in [new_lo, new_hi]
    as a random tree (chain: one behind the other)."""
    Hq, Hkv, d = heads
    return dict(name=name, op=op, n=n, ctx_lo=ctx_lo, ctx_hi=ctx_hi, skew=skew, new_lo=new_lo, new_hi=new_hi, Hq=Hq,
                Hkv=Hkv, d=d, cache=cache, chain=chain, page=page, structure=structure)


def listed():
    return [
        # interactive decode: the next tokens of four users, an 8B-shaped layer; latency bound
        _rope("rope_4users", 4, (32, 8, 128), 128),
        # a batch of prompts of the same layer
        _rope("rope_prompts_8b", 22011, (32, 8, 128), 128),
        # prompts with images and video, a 70B-shaped layer: positions in time, height and width, fp32 projections
        _rope("rope_video_70b", 8190, (64, 8, 128), 128, axes=3, dtype="f32"),
        # a few short prompts go into an empty cache and are read back for their attention
        _cache("cache_short_prompts", 4, 0, 0, 16, 512, (8, 64)),
        # chunked prefill: chunks of 512..2048 tokens behind contexts of up to 16384 tokens
        _cache("cache_chunks", 32, 0, 16384, 512, 2048, (8, 128)),
        # interactive decode, one token of each of four users: the smallest attention
        _tree("single_4users", "tree", 4, 300, 3000, 1, 1, (32, 8, 128), structure=3),
        # a large decode batch of very different lengths, one token each
        _tree("single_256", "tree", 256, 32, 16384, 1, 1, (32, 8, 128), skew=3),
        # drafted trees of a small batch, an 8B-shaped layer
        _tree("drafts_8b", "tree", 16, 500, 4000, 5, 24, (32, 8, 128)),
        # drafted trees of up to 64 tokens, a 70B-shaped layer and a large batch: the most arithmetic
        _tree("drafts_70b", "tree", 64, 512, 8192, 33, 64, (64, 8, 128)),
        # two very long documents, short chains drafted from the text itself, cache in bf16, head dimension 64
        _tree("chains_long_d64", "tree", 2, 65536, 131072, 3, 9, (64, 8, 64), cache="bf16", chain=True, page=64),
        # a whole step of one layer for four users
        _tree("step_4users", "step", 4, 300, 3000, 4, 16, (32, 8, 128), structure=5),
        # a whole step of one layer for a batch
        _tree("step_128", "step", 128, 128, 4096, 4, 12, (32, 8, 128)),
    ]


HEADS = [(32, 8, 128), (32, 8, 128), (64, 8, 128), (64, 8, 128), (8, 8, 64), (64, 8, 64), (8, 2, 128), (4, 1, 128), (16, 2, 128),
         (16, 16, 128), (28, 4, 128), (40, 8, 64)]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _draw_once(rng):
    heads = rng.choice(HEADS)
    op = rng.choice(["rope", "rope", "cache", "cache", "tree", "tree", "tree", "tree", "step", "step"])
    s = rng.randrange(1 << 20)
    page = rng.choice([16, 16, 16, 32, 64, 128, 48])
    cache = rng.choice(["f8", "f8", "f8", "bf16"])
    if op == "rope":
        d = heads[2]
        c = _rope("", _log(rng, 1, 32768), heads, rng.choice([d, d, d // 2, 32, 0]), rng.choice([1, 1, 2, 3]), rng.random() < 0.3,
                  rng.random() < 0.8, rng.choice(["bf16", "bf16", "f32"]), rng.choice(["bf16", "bf16", "f32"]), s)
        if c["rot"] == 0:
            c["axes"], c["interleaved"] = 1, False
            c["norm"] = True
        return c
    if op == "cache":
        n = _log(rng, 1, 64)
        new_hi = max(1, min(4096, _log(rng, 1, 60000) // n))
        ctx_hi = rng.choice([0, max(1, min(32768, _log(rng, 100, 400000) // n))])
        return _cache("", n, ctx_hi // rng.choice([2, 50]), ctx_hi, max(1, new_hi // rng.choice([1, 4, 16])), new_hi, heads[1:], cache,
                      rng.choice(["bf16", "bf16", "f32"]), rng.choice(["bf16", "bf16", "f32"]), page, s)
    n = _log(rng, 1, 300)
    new_hi = rng.choice([1, 1, _log(rng, 2, 64), _log(rng, 2, 64)])
    ctx_hi = max(1, min(131072, _log(rng, 200, 600000) // n))
    return _tree("", op, n, ctx_hi // rng.choice([2, 10, 1000]), ctx_hi, max(1, new_hi // rng.choice([1, 2, 16])), new_hi, heads, cache,
                 rng.random() < 0.3, rng.choice([1, 1, 3]), page, s)


def _padded_bytes(case):
    """What the plain form's padded keys and values take, 32 bits each."""
    if case["op"] not in ("tree", "step"):
        return 0
    ctx, new = _lengths(case)
    longest, T = int((ctx + new).max()), int(new.max())
    return 4 * case["n"] * longest * (2 * case["Hkv"] * case["d"] + 2 * T * case["Hq"])


def _cost(case):
    w = work(case)
    return w["bytes"] / 5e12 + w["flops"] / 6e14


def draw(rng):
    while True:
        c = _draw_once(rng)
        c.pop("name", None)
        if _cost(c) <= 0.5e-3 and _padded_bytes(c) <= 20 << 30:      # under the largest listed case
            return c


# ---------------------------------------------------------------------------------------------
# structure of a case (lengths, trees, slots): the same for every seed
# ---------------------------------------------------------------------------------------------

def _lengths(case):
    """(context, new tokens) of every request."""
    rng = np.random.default_rng(case["structure"] + 1)
    n = case["n"]
    ctx = case["ctx_lo"] + np.floor((case["ctx_hi"] + 1 - case["ctx_lo"]) * rng.random(n) ** case["skew"]).astype(np.int64)
    return ctx, rng.integers(case["new_lo"], case["new_hi"] + 1, size=n)


def _tables(case):
    """(block table, blocks of the pool, slot of every new token): a seeded random placement of the pages."""
    rng = np.random.default_rng(case["structure"] + 2)
    ctx, new = _lengths(case)
    page = case["page"]
    blocks = (ctx + new + page - 1) // page
    pool = int(blocks.sum() * 1.1) + 2
    perm = rng.permutation(pool)
    table = np.zeros((case["n"], int(blocks.max())), np.int32)
    at = 0
    for i, b in enumerate(blocks):
        table[i, :b] = perm[at:at + b]
        at += b
    req = np.repeat(np.arange(case["n"]), new)
    pos = np.concatenate([np.arange(c, c + t) for c, t in zip(ctx, new)])
    return table, pool, table[req, pos // page].astype(np.int64) * page + pos % page


def _trees(case):
    """(parent of every drafted token or -1, ancestor bits, depth, accepted tokens [n][T], their number)."""
    rng = np.random.default_rng(case["structure"] + 3)
    _, new = _lengths(case)
    bits, depth, keep, count = [], [], np.zeros((case["n"], int(new.max())), np.int32), []
    for i, T in enumerate(new):
        par, own_bits, own_depth = [], [], []
        for t in range(T):
            p = t - 1 if case["chain"] or t == 0 else int(rng.integers(0, t)) if rng.random() < 0.7 else t - 1
            par.append(p)
            own_bits.append((1 << t) | (own_bits[p] if p >= 0 else 0))
            own_depth.append(own_depth[p] + 1 if p >= 0 else 0)
        bits += own_bits
        depth += own_depth
        path, t = [], int(rng.integers(0, T))          # the accepted branch: the ancestors of a random token
        while t >= 0:
            path.append(t)
            t = par[t]
        path = path[::-1]
        keep[i, :len(path)] = path
        count.append(len(path))
    as_int64 = np.array([b - (1 << 64) if b >> 63 else b for b in bits], np.int64)
    return as_int64, np.array(depth), keep, np.array(count, np.int32)


def _pair_axis(case):
    """Axis of every rotated pair: contiguous sections, the first a quarter of the pairs, the others even."""
    pairs, axes = case["rot"] // 2, case["axes"]
    if axes == 1:
        return [0] * pairs
    first = pairs // 4 if axes > 2 else pairs // 2
    cuts = [first + (pairs - first) * a // (axes - 1) for a in range(axes)]
    return [int(np.searchsorted(cuts, p, side="right")) for p in range(pairs)]


# ---------------------------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------------------------

def _type(name):
    return {"bf16": torch.bfloat16, "f32": torch.float32}[name]


def _rows(gen, tokens, heads, d, outlier=0.0):
    """N(0, 1) rows; some channels of every head larger, as keys have them."""
    x = torch.randn(tokens, heads, d, generator=gen, device=DEV)
    if outlier:
        x *= 1 + outlier * (torch.rand(heads, d, generator=gen, device=DEV) < 0.03)
    return x


def _table(max_pos, rot):
    """[max_pos][2][rot / 2]: cosines, sines."""
    if rot == 0:
        return None
    freq = 10000.0 ** (-torch.arange(0, rot, 2, dtype=torch.float64, device=DEV) / rot)
    angle = torch.arange(max_pos, dtype=torch.float64, device=DEV)[:, None] * freq
    return torch.stack([angle.cos(), angle.sin()], dim=1).float().contiguous()


def _pool(case, gen, blocks):
    Hkv, d, page = case["Hkv"], case["d"], case["page"]
    k = _rows(gen, blocks * page, Hkv, d, 4.0).view(blocks, page, Hkv, d).transpose(1, 2)
    v = _rows(gen, blocks * page, Hkv, d).view(blocks, page, Hkv, d).transpose(1, 2)
    by_four = lambda x: x.reshape(blocks, Hkv, page // 4, 4, d).transpose(-1, -2).contiguous()  # noqa: E731
    if case["cache"] == "bf16":
        return k.to(torch.bfloat16).contiguous(), by_four(v.to(torch.bfloat16)), None
    (kc, ks), (vc, vs) = _quantize(k), _quantize(v)
    scales = torch.stack([ks, vs], dim=2).contiguous().view(torch.float8_e8m0fnu)
    return kc.contiguous().view(torch.float8_e4m3fn), by_four(vc).view(torch.float8_e4m3fn), scales


def prepare(case, seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(int(seed))
    dev = lambda x, t=None: torch.from_numpy(np.ascontiguousarray(x)).to(DEV, t)  # noqa: E731
    s = dict(case=case, op=case["op"])
    d, Hkv = case["d"], case["Hkv"]
    if case["op"] == "rope":
        tokens, Hq, dtype = case["tokens"], case["Hq"], _type(case["dtype"])
        # queries, keys and values of a token side by side, as the projection leaves them
        qkv = torch.randn(tokens, Hq + 2 * Hkv, d, generator=gen, device=DEV).to(dtype)
        s["q"], s["k"] = qkv[:, :Hq], qkv[:, Hq:Hq + Hkv]
        max_pos = 40000
        s["positions"] = torch.randint(0, max_pos, (case["axes"], tokens), generator=gen, device=DEV, dtype=torch.int32)
        s["table"], s["pair_axis"] = _table(max_pos, case["rot"]), _pair_axis(case)
        s["axis_index"] = torch.tensor(s["pair_axis"], device=DEV)
        s["wq"], s["wk"] = ((1 + 0.1 * torch.randn(d, generator=gen, device=DEV)).to(dtype) if case["norm"] else None for _ in "qk")
        s["q_out"], s["k_out"] = (torch.empty(tokens, h, d, dtype=_type(case["out"]), device=DEV) for h in (Hq, Hkv))
    else:
        ctx, new = _lengths(case)
        table, blocks, slots = _tables(case)
        s["pool"] = _pool(case, gen, blocks)
        s["block_table"], s["slots"] = dev(table), dev(slots)
        s["lens"] = dev(ctx + new, torch.int32)
        s["longest"], s["page"], s["total_new"] = int((ctx + new).max()), case["page"], int(new.sum())
    if case["op"] == "cache":
        rows = int((ctx + new).sum())
        s["k"] = _rows(gen, s["total_new"], Hkv, d, 4.0).to(_type(case["dtype"]))
        s["v"] = _rows(gen, s["total_new"], Hkv, d).to(_type(case["dtype"]))
        s["start"] = dev(np.cumsum(ctx + new) - (ctx + new), torch.int32)
        req = np.repeat(np.arange(case["n"]), ctx + new)
        pos = np.concatenate([np.arange(x) for x in ctx + new])
        s["all_slots"] = dev(table[req, pos // case["page"]].astype(np.int64) * case["page"] + pos % case["page"])
        s["k_out"], s["v_out"] = (torch.empty(rows, Hkv, d, dtype=_type(case["out"]), device=DEV) for _ in "kv")
    if case["op"] in ("tree", "step"):
        bits, depth, keep, count = _trees(case)
        q_start = np.concatenate([[0], np.cumsum(new)])
        s["q_start"], s["max_q"] = dev(q_start, torch.int32), int(new.max())
        s["row_req"], s["row_t"] = dev(np.repeat(np.arange(case["n"]), new)), dev(np.concatenate([np.arange(x) for x in new]))
        s["mask"] = None if case["chain"] else dev(bits)
        s["bits"] = dev(bits)
        s["out"] = torch.empty(s["total_new"], case["Hq"], d, dtype=torch.bfloat16, device=DEV)
        s["scale"] = 1.0 / math.sqrt(d)
        s["q"] = _rows(gen, s["total_new"], case["Hq"], d).to(torch.bfloat16)
    if case["op"] == "step":
        Hq = case["Hq"]
        qkv = _rows(gen, s["total_new"], Hq + 2 * Hkv, d).to(torch.bfloat16)
        s["q_in"], s["k"], s["v"] = qkv[:, :Hq], qkv[:, Hq:Hq + Hkv], qkv[:, Hq + Hkv:]
        s["wq"], s["wk"] = ((1 + 0.1 * torch.randn(d, generator=gen, device=DEV)).to(torch.bfloat16) for _ in "qk")
        s["table"], s["pair_axis"], s["axis_index"] = _table(s["longest"], d), None, torch.zeros(d // 2, dtype=torch.int64, device=DEV)
        s["positions"] = dev(np.repeat(ctx, new) + depth, torch.int32)[None]
        s["keep"], s["count"], s["new_lens"] = dev(keep), dev(count), torch.empty_like(s["lens"])
    if own:
        # what a serving program keeps from call to call: the cache, the rotation of this batch, a workspace
        from paper_2602_06072_amd import binding as pk
        s["pk"] = pk
        if "pool" in s:
            s["cache"] = pk.KvCache(*s["pool"])
        if "table" in s:
            s["rope"] = None if s["table"] is None else pk.Rope(s["table"], s["positions"], s["pair_axis"], case.get("interleaved", False))
        if case["op"] in ("tree", "step"):
            s["ws"] = pk.new_tree_workspace(case["n"], s["max_q"], case["Hq"], Hkv, d)
    return s


# ---------------------------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------------------------

def run(s):
    return (_run_own if own else _run_plain)(s)


def _run_own(s):
    pk, op = s["pk"], s["op"]
    if op == "rope":
        pk.qk_norm_rope(s["q"], s["k"], s["q_out"], s["k_out"], s["wq"], s["wk"], EPS, s["rope"])
        return s["q_out"], s["k_out"]
    if op == "cache":
        pk.kv_cache_write(s["cache"], s["k"], s["v"], s["slots"])
        pk.kv_cache_read(s["cache"], s["block_table"], s["lens"], s["start"], s["k_out"], s["v_out"])
        return s["k_out"], s["v_out"]
    if op == "step":
        pk.qkv_cache_write(s["cache"], s["q_in"], s["k"], s["v"], s["slots"], s["q"], s["wq"], s["wk"], EPS, s["rope"])
    pk.tree_attn(s["cache"], s["q"], s["q_start"], s["max_q"], s["mask"], s["block_table"], s["lens"], s["out"], s["scale"], s["ws"])
    if op == "tree":
        return s["out"]
    pk.kv_cache_keep(s["cache"], s["block_table"], s["lens"], s["q_start"], s["max_q"], s["keep"], s["count"], s["new_lens"])
    return _step_outputs(s)


def _step_outputs(s):
    k, v, scales = s["pool"]
    return {"out": s["out"], "k": k, "v": v, "lens": s["new_lens"], **({} if scales is None else {"scales": scales})}


# ------------------------------------------------------------------ the plain form

def _norm(x, w):
    x = x.float()
    return x if w is None else x * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS) * w.float()


def _cos_sin(table, positions, axis_index):
    """[tokens][1][pairs] each: every pair from the row of its own axis' position."""
    pairs = torch.arange(table.shape[2], device=table.device)
    at = positions.long().t()[:, axis_index]                       # [tokens][pairs]
    return table[at, 0, pairs][:, None], table[at, 1, pairs][:, None]


def _rotate(x, cos, sin, interleaved):
    rot = 2 * cos.shape[-1]
    y = x[..., :rot]
    a, b = (y[..., 0::2], y[..., 1::2]) if interleaved else (y[..., :rot // 2], y[..., rot // 2:])
    a, b = a * cos - b * sin, b * cos + a * sin
    y = torch.stack([a, b], dim=-1).flatten(-2) if interleaved else torch.cat([a, b], dim=-1)
    return torch.cat([y, x[..., rot:]], dim=-1)


def _quantize(x):
    """(codes, exponents + 127) as bytes; rows are the last axis."""
    x = x.float()
    largest = torch.where(torch.isfinite(x), x.abs(), torch.zeros_like(x)).amax(-1)
    m, e = torch.frexp(largest)                                    # largest = m 2^e, 448 = 0.875 * 2^9
    E = torch.where(largest > 0, e - 9 + (m > 0.875).to(e.dtype), torch.full_like(e, -126)).clamp(-126, 127)
    factor = ((127 - E) << 23).to(torch.int32).view(torch.float32)     # 2^-E from its bits
    return (x * factor[..., None]).to(torch.float8_e4m3fn).view(torch.uint8), (E + 127).to(torch.uint8)


def _put(pool, slots, page, k, v):
    """Writes rows (f32, [tokens][Hkv][d]) to their slots."""
    blk, off = slots // page, slots % page
    kp, vp, scales = pool
    if scales is None:
        kp[blk, :, off] = k.to(torch.bfloat16)
        vp[blk, :, off // 4, :, off % 4] = v.to(torch.bfloat16)
        return
    (kc, ks), (vc, vs) = _quantize(k), _quantize(v)
    kp.view(torch.uint8)[blk, :, off] = kc
    vp.view(torch.uint8)[blk, :, off // 4, :, off % 4] = vc
    scales.view(torch.uint8)[blk, :, 0, off] = ks
    scales.view(torch.uint8)[blk, :, 1, off] = vs


def _take(pool, slots, page):
    """Rows (f32, [...][Hkv][d]) of slots [...]."""
    blk, off = slots // page, slots % page
    kp, vp, scales = pool
    if scales is None:
        return kp[blk, :, off].float(), vp[blk, :, off // 4, :, off % 4].float()
    k = kp.view(torch.uint8)[blk, :, off].view(torch.float8_e4m3fn).float()
    v = vp.view(torch.uint8)[blk, :, off // 4, :, off % 4].view(torch.float8_e4m3fn).float()
    ks, vs = (scales.view(torch.uint8)[blk, :, i, off].view(torch.float8_e8m0fnu).float()[..., None] for i in (0, 1))
    return k * ks, v * vs


def _attend(q, s):
    """q: [rows][Hq][d] in f32.  Keys and values of all requests side by side, padded to the longest."""
    lens, page, n = s["lens"].long(), s["page"], s["lens"].shape[0]
    Hq, d = q.shape[1:]
    pos = torch.arange(s["longest"], device=q.device)
    slots = s["block_table"].long()[:, pos // page] * page + pos % page
    k, v = _take(s["pool"], slots, page)                           # [n][L][Hkv][d]
    k, v = k.transpose(1, 2), v.transpose(1, 2)
    Hkv, T = k.shape[1], s["max_q"]
    new = s["q_start"][1:].long() - s["q_start"][:-1].long()
    rows = (s["q_start"][:-1].long()[:, None] + torch.arange(T, device=q.device)).clamp(max=q.shape[0] - 1)
    x = q[rows].view(n, T, Hkv, Hq // Hkv, d).permute(0, 2, 1, 3, 4).reshape(n, Hkv, -1, d)
    scores = (torch.matmul(x, k.transpose(-1, -2)) * s["scale"]).view(n, Hkv, T, Hq // Hkv, -1)
    drafted = pos - (lens - new)[:, None]                          # [n][L]: number of the drafted token, negative in the context
    bit = (s["bits"][rows][:, :, None] >> drafted.clamp(0, 63)[:, None]) & 1
    seen = ((drafted < 0)[:, None] | (bit != 0)) & (pos < lens[:, None])[:, None]          # [n][T][L]
    scores = scores.masked_fill(~seen[:, None, :, None], -math.inf)
    top = scores.amax(-1, keepdim=True)
    p = torch.exp(scores - torch.where(top == -math.inf, torch.zeros_like(top), top))
    total = p.sum(-1, keepdim=True)
    p = p / torch.where(total > 0, total, torch.ones_like(total))
    o = torch.matmul(p.view(n, Hkv, -1, p.shape[-1]), v).view(n, Hkv, T, Hq // Hkv, d)
    return o.permute(0, 2, 1, 3, 4).reshape(n, T, Hq, d)[s["row_req"], s["row_t"]]


def _run_plain(s):
    op = s["op"]
    if op in ("rope", "step"):
        q, k = _norm(s["q"] if op == "rope" else s["q_in"], s["wq"]), _norm(s["k"], s["wk"])
        if s["table"] is not None:
            cos, sin = _cos_sin(s["table"], s["positions"], s["axis_index"])
            interleaved = s["case"].get("interleaved", False)
            q, k = _rotate(q, cos, sin, interleaved), _rotate(k, cos, sin, interleaved)
    if op == "rope":
        return q.to(s["q_out"].dtype), k.to(s["k_out"].dtype)
    if op == "cache":
        _put(s["pool"], s["slots"], s["page"], s["k"].float(), s["v"].float())
        k, v = _take(s["pool"], s["all_slots"], s["page"])
        return k.to(s["k_out"].dtype), v.to(s["v_out"].dtype)
    if op == "step":
        _put(s["pool"], s["slots"], s["page"], k, s["v"].float())
        q = q.to(torch.bfloat16)
    else:
        q = s["q"]
    s["out"] = _attend(q.float(), s).to(torch.bfloat16)
    if op == "tree":
        return s["out"]
    # the accepted tokens: read, then written behind the context
    base = s["lens"].long() - (s["q_start"][1:] - s["q_start"][:-1]).long()
    j = torch.arange(s["keep"].shape[1], device=DEV)
    req, at = torch.nonzero(j < s["count"][:, None], as_tuple=True)
    page, table = s["page"], s["block_table"].long()
    src, dst = (table[req, x // page] * page + x % page for x in (base[req] + s["keep"].long()[req, at], base[req] + at))
    kp, vp, scales = s["pool"]
    as_bytes = lambda x: x.view(torch.uint8) if x.element_size() == 1 else x  # noqa: E731
    kp, vp = as_bytes(kp), as_bytes(vp)
    old = [kp[src // page, :, src % page], vp[src // page, :, src % page // 4, :, src % 4]]
    if scales is not None:
        old.append(as_bytes(scales)[src // page, :, :, src % page])
        as_bytes(scales)[dst // page, :, :, dst % page] = old[2]
    kp[dst // page, :, dst % page] = old[0]
    vp[dst // page, :, dst % page // 4, :, dst % 4] = old[1]
    s["new_lens"] = (base + s["count"]).to(torch.int32)
    return _step_outputs(s)


# ---------------------------------------------------------------------------------------------
# what a pass cannot do without
# ---------------------------------------------------------------------------------------------

def work(case):
    size = {"bf16": 2, "f32": 4, "f8": 1}
    Hkv, d = case["Hkv"], case["d"]
    if case["op"] == "rope":
        values = case["tokens"] * (case["Hq"] + Hkv) * d
        distinct = min(case["tokens"] * case["axes"], 40000)       # rows of the table
        return {"bytes": values * (size[case["dtype"]] + size[case["out"]]) + distinct * case["rot"] * 4 // max(1, case["axes"]) + 4 * case["axes"] * case["tokens"],
                "flops": 10 * values}
    ctx, new = _lengths(case)
    total, fresh = int((ctx + new).sum()), int(new.sum())
    row = 2 * Hkv * (d * size[case["cache"]] + (1 if case["cache"] == "f8" else 0))      # K and V of a token in the cache
    if case["op"] == "cache":
        return {"bytes": fresh * (2 * Hkv * d * size[case["dtype"]] + row + 8) + total * (row + 2 * Hkv * d * size[case["out"]]),
                "flops": 4 * (fresh + total) * Hkv * d}
    Hq = case["Hq"]
    bits = _trees(case)[0]
    pairs = int((ctx * new).sum()) + sum(bin(int(b) & 0xFFFFFFFFFFFFFFFF).count("1") for b in bits)
    w = {"bytes": total * row + 2 * fresh * Hq * d * 2 + 8 * fresh + 4 * total // case["page"], "flops": 4 * d * Hq * pairs}
    if case["op"] == "step":
        # projections in, drafted rows into the cache (their reading is counted above), accepted rows moved
        w["bytes"] += fresh * ((Hq + 2 * Hkv) * d * 2 + row + d * 4) + 2 * int(_trees(case)[3].sum()) * row
    return w


# ---------------------------------------------------------------------------------------------
# the definition, in 64 bits
# ---------------------------------------------------------------------------------------------

def _value_of_byte():
    """Value of every E4M3 byte: sign, 4 exponent bits (bias 7), 3 fraction bits; 0x7F and 0xFF are no numbers."""
    out = []
    for b in range(256):
        e, f = b >> 3 & 15, b & 7
        x = math.nan if b & 127 == 127 else f / 8 * 2.0 ** -6 if e == 0 else (1 + f / 8) * 2.0 ** (e - 7)
        out.append(-x if b & 128 else x)
    return torch.tensor(out, dtype=torch.float64, device=DEV)


def _power(E):
    """2^E in 64 bits, from its bits."""
    return (E.to(torch.int64) + 1023 << 52).view(torch.float64)


def _nearest_e4m3(x):
    """The multiple of 2^E that E4M3 with the row's scale has next to x (ties to the even one), and 2^E."""
    top = x.abs().amax(-1, keepdim=True)
    E = torch.frexp(top)[1] - 9                                    # 448 * 2^E is 0.875 of the next power of two
    E = torch.where(top > F8_MAX * _power(E), E + 1, E).clamp(-126, 127)
    y = x * _power(-E)
    step = _power(torch.frexp(y.abs().clamp(min=2.0 ** -6))[1] - 4)
    return torch.round(y / step) * step, _power(E)


def exact(case, seed):
    s = prepare(case, seed)
    op, d, Hkv = case["op"], case["d"], case["Hkv"]

    def turned(x, w):
        x = x.double()
        if w is not None:
            x = x / torch.sqrt((x ** 2).sum(-1, keepdim=True) / d + EPS) * w.double()
        if s["table"] is None:
            return x
        h = s["table"].shape[2]
        out = x.clone()
        for p in range(h):
            i, j = (2 * p, 2 * p + 1) if case.get("interleaved") else (p, p + h)
            row = s["table"][s["positions"][int(s["axis_index"][p])].long()]
            c, n = row[:, 0, p].double()[:, None], row[:, 1, p].double()[:, None]
            out[..., i] = x[..., i] * c - x[..., j] * n
            out[..., j] = x[..., i] * n + x[..., j] * c
        return out

    if op == "rope":
        return turned(s["q"], s["wq"]), turned(s["k"], s["wk"])
    byte_value = _value_of_byte() if case["cache"] == "f8" else None
    page = case["page"]

    def codes_and_scales():
        """The cache token by token: codes [slots][Hkv][d] of K and V, scales [slots][Hkv] of both, in 64 bits."""
        kp, vp, sc = s["pool"]
        look = (lambda x: byte_value[x.view(torch.uint8).long()]) if byte_value is not None else (lambda x: x.double())
        k = look(kp).transpose(1, 2).reshape(-1, Hkv, d)
        v = look(vp).permute(0, 2, 4, 1, 3).reshape(-1, Hkv, d)
        if sc is None:
            return k, v, torch.ones(k.shape[0], Hkv, 2, dtype=torch.float64, device=DEV)
        return k, v, _power(sc.view(torch.uint8).long() - 127).permute(0, 3, 1, 2).reshape(-1, Hkv, 2)

    if 30 * s["pool"][0].numel() > 120e9:
        return None
    k, v, sc = codes_and_scales()
    if op in ("cache", "step"):
        kn, vn = (s["k"].double() if op == "cache" else turned(s["k"], s["wk"])), s["v"].double()
        if byte_value is not None:
            for i, (dst, x) in enumerate(((k, kn), (v, vn))):
                code, scale = _nearest_e4m3(x)
                dst[s["slots"]], sc[s["slots"], :, i] = code, scale[..., 0]
        else:
            k[s["slots"]], v[s["slots"]] = kn.to(torch.bfloat16).double(), vn.to(torch.bfloat16).double()
    if op == "cache":
        return k[s["all_slots"]] * sc[s["all_slots"], :, 0, None], v[s["all_slots"]] * sc[s["all_slots"], :, 1, None]
    ctx, new = _lengths(case)
    table = s["block_table"].long()
    q = s["q"].double() if op == "tree" else turned(s["q_in"], s["wq"]).to(torch.bfloat16).double()
    out = torch.zeros(q.shape, dtype=torch.float64, device=DEV)
    r, at = case["Hq"] // Hkv, 0
    for i in range(case["n"]):
        c, T = int(ctx[i]), int(new[i])
        pos = torch.arange(c + T, device=DEV)
        slot = table[i, pos // page] * page + pos % page
        ki, vi = ((x[slot] * sc[slot, :, a, None]).transpose(0, 1).contiguous() for a, x in ((0, k), (1, v)))      # [Hkv][L][d]
        seen = torch.ones(T, c + T, dtype=torch.bool, device=DEV)
        word = s["bits"][at:at + T]
        for j in range(T):
            seen[:, c + j] = word >> j & 1 != 0
        x = q[at:at + T].reshape(T, Hkv, r, d).permute(1, 0, 2, 3).reshape(Hkv, T * r, d).contiguous()
        w = torch.bmm(x, ki.transpose(1, 2).contiguous()) * s["scale"]
        w = w.view(Hkv, T, r, -1).masked_fill(~seen[None, :, None], -math.inf).softmax(-1).view(Hkv, T * r, -1)
        out[at:at + T] = torch.bmm(w, vi).view(Hkv, T, r, d).permute(1, 0, 2, 3).reshape(T, Hkv * r, d)
        at += T
    if op == "tree":
        return out
    keep, count = s["keep"].cpu().numpy(), s["count"].cpu().numpy()
    for i in range(case["n"]):
        src = torch.tensor([int(ctx[i]) + int(x) for x in keep[i, :count[i]]], device=DEV)
        dst = torch.arange(int(ctx[i]), int(ctx[i]) + int(count[i]), device=DEV)
        src, dst = (table[i, x // page] * page + x % page for x in (src, dst))
        for x in (k, v, sc):
            x[dst] = x[src]
    blocks = s["pool"][0].shape[0]
    res = {"out": out, "k": k.view(blocks, page, Hkv, d).transpose(1, 2), "lens": None,
           "v": v.view(blocks, page // 4, 4, Hkv, d).permute(0, 3, 1, 4, 2)}
    if byte_value is not None:
        res["scales"] = sc.view(blocks, page, Hkv, 2).permute(0, 2, 3, 1)
    return res
