"""Cases for timing the operators around branching and drafted decoding on one GPU: attention over a paged cache whose
requests share the pages of a prefix, the pages themselves (forking, reserving, compacting, copying), and the judging of drafted
tokens from given random numbers.

listed() and draw() give cases, prepare() makes what a serving program has in hand before the call, run() makes
one pass and work() states what a pass cannot do without.  exact() computes the results in 64 bits from the
definitions.  With `own` false, run() is the plain form of the operators in elementary operations; with `own` true it
calls paper_2602_06072_amd.binding.

The lengths of a case come from its own "structure" number, so that work() knows them; values come from the seed.

op       one pass is
shared   shared_tree_attn: attention of the new tokens of every request; the requests of a family have the pages of a prefix
         in common
fork     kv_pages_select (every request becomes some), kv_pages_reserve (pages for their new tokens; a shared page that would be
         written is replaced by a copy), kv_cache_copy of those pages, kv_pages_select (one of each stays)
compact  kv_pages_compact (the pages in use get the lowest numbers), kv_cache_copy of the pages that move
verify   draft_verify: which drafted tokens stay, and the token behind them; one token a request: plain sampling

The cache (types "f8" and "bf16"): K [blocks][Hkv][page][d]; V [blocks][Hkv][page / 4][d][4], four tokens
interleaved; with "f8" E4M3 codes and scales [blocks][Hkv][2][page] (K, V), powers of two, one for each token and
head.  The pages of a batch: block table [n][max_blocks], lengths [n], pages that each request holds [n], and for every block of the
pool how many of these hold it.

Judging.  Row t of a request's logits is the distribution of the token behind its token t: weights exp((l - max l) / temperature)
over their sum; a NaN counts as -inf.  Token 0 stays.  The parent of token t is its highest lower ancestor in its mask word.  Tokens are looked at by
rising number, each whose parent is the last one that stayed: with target P and draft Q of the parent, after k refused children c_k, Z_k
(c_0 = 0, Z_0 = 1) token x stays if P(x) > (c_k + u Z_k) Q(x); refused, c_{k+1} = c_k + Z_k and Z_{k+1} is the sum of max(P - c_{k+1} Q, 0).
Without draft logits drafted tokens are no draws: x stays if P(x) > u Z_k, and its probability leaves P if not.  The token behind the last
one that stayed is the first whose cumulative weight in what is left of P is over u times the whole.  Temperature 0: the first of the largest logits.
"""
import math

import numpy as np
import torch

own = False
DEV = "cuda"
F8_MAX = 448.0


# ---------------------------------------------------------------------------------------------
# cases
# ---------------------------------------------------------------------------------------------

def _shared(name, families, members_lo, members_hi, prefix_lo, prefix_hi, own_lo, own_hi, new_lo, new_hi, heads, cache="f8", chain=True, page=16,
            structure=0):
    """Families of requests with a prefix in [prefix_lo, prefix_hi], of which whole pages are shared, own tokens in
    [own_lo, own_hi] behind it, new tokens in [new_lo, new_hi]."""
    Hq, Hkv, d = heads
    return dict(name=name, op="shared", families=families, members_lo=members_lo, members_hi=members_hi, prefix_lo=prefix_lo, prefix_hi=prefix_hi,
                own_lo=own_lo, own_hi=own_hi, new_lo=new_lo, new_hi=new_hi, Hq=Hq, Hkv=Hkv, d=d, cache=cache, chain=chain, page=page,
                structure=structure)


def _fork(name, n, kids_lo, kids_hi, ctx_lo, ctx_hi, grow_lo, grow_hi, heads, cache="f8", page=16, spare=1.5, structure=0):
    """n requests with a context in [ctx_lo, ctx_hi], each becoming [kids_lo, kids_hi] that grow by [grow_lo, grow_hi] tokens;
    spare: blocks of the pool over those that are asked for (below 1 the last requests may get none)."""
    Hkv, d = heads
    return dict(name=name, op="fork", n=n, kids_lo=kids_lo, kids_hi=kids_hi, ctx_lo=ctx_lo, ctx_hi=ctx_hi, grow_lo=grow_lo, grow_hi=grow_hi, Hkv=Hkv,
                d=d, cache=cache, page=page, spare=spare, structure=structure)


def _compact(name, n, ctx_lo, ctx_hi, heads, used, cache="f8", page=16, structure=0):
    """n requests with a context in [ctx_lo, ctx_hi] whose pages are strewn over a pool of which they are the part `used`."""
    Hkv, d = heads
    return dict(name=name, op="compact", n=n, ctx_lo=ctx_lo, ctx_hi=ctx_hi, Hkv=Hkv, d=d, cache=cache, page=page, used=used, structure=structure)


def _verify(name, n, new_lo, new_hi, vocab, dtype="bf16", draft=True, tree=False, greedy=0.0, structure=0):
    """n requests with [new_lo, new_hi] tokens, the first one given, the others drafted (a random tree or one behind the
    other); draft: with the logits they were drawn from.  greedy: part of the requests with temperature 0."""
    return dict(name=name, op="verify", n=n, new_lo=new_lo, new_hi=new_hi, vocab=vocab, dtype=dtype, draft=draft, tree=tree, greedy=greedy,
                structure=structure)


def listed():
    return [
        # eight answers drawn from one prompt, the smallest call: latency bound
        _shared("samples_8", 1, 8, 8, 1200, 1200, 1, 200, 1, 1, (32, 8, 128)),
        # a system prompt in front of a whole decode batch
        _shared("prompt_128", 1, 128, 128, 8200, 8200, 16, 1024, 1, 1, (32, 8, 128)),
        # documents that are asked about by several users each, drafted trees, a 70B-shaped layer
        _shared("families_70b", 16, 4, 12, 1024, 8192, 16, 600, 4, 16, (64, 8, 128), chain=False),
        # two long documents, short chains drafted from the text itself, cache in bf16, head dimension 64
        _shared("documents_d64", 2, 9, 16, 40000, 66000, 20, 300, 3, 5, (64, 8, 64), cache="bf16", page=64),
        # four prompts are answered twice each: page tables and a few copies, latency bound
        _fork("fork_4", 4, 2, 2, 100, 2000, 1, 1, (8, 128)),
        # best of several for a batch, with room for drafted tokens
        _fork("fork_64", 64, 2, 8, 200, 6000, 4, 40, (8, 128)),
        # a small pool of a bf16 cache after its first requests have left
        _compact("compact_small", 6, 100, 3000, (8, 64), 0.4, cache="bf16", page=32),
        # a large pool in which half of the pages are free, strewn all over: the most bytes
        _compact("compact_large", 300, 200, 5000, (8, 128), 0.5),
        # the next token of four users: the smallest sampling
        _verify("sample_4users", 4, 1, 1, 32000),
        # chains of drafted tokens of a batch with a small draft model of the same vocabulary, some users greedy
        _verify("chains_64", 64, 4, 8, 128256, greedy=0.2),
        # drafted trees of a small batch, fp32 logits
        _verify("trees_16", 16, 16, 48, 32000, dtype="f32", tree=True),
        # tokens drafted from the text itself, a vocabulary of odd size: rows at every alignment
        _verify("lookup_200", 200, 2, 6, 50257, draft=False, greedy=0.1),
    ]


HEADS = [(32, 8, 128), (32, 8, 128), (64, 8, 128), (8, 8, 64), (64, 8, 64), (8, 2, 128), (4, 1, 128), (16, 2, 128), (16, 16, 128), (28, 4, 128),
         (40, 8, 64)]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _draw_once(rng):
    op = rng.choice(["shared", "shared", "shared", "fork", "compact", "verify", "verify", "verify"])
    s = rng.randrange(1 << 20)
    heads = rng.choice(HEADS)
    cache = rng.choice(["f8", "f8", "f8", "bf16"])
    page = rng.choice([16, 16, 16, 32, 64, 128, 48])
    if op == "shared":
        families = _log(rng, 1, 24)
        members = max(1, _log(rng, 2, 256) // families)
        prefix = max(1, _log(rng, 60, 200000) // max(families, members // 2))
        own_hi = max(1, min(4096, _log(rng, 16, 100000) // (families * members)))
        new = rng.choice([1, 1, _log(rng, 2, 64), _log(rng, 2, 24)])
        return _shared("", families, max(1, members // rng.choice([1, 2, 3])), members, prefix // rng.choice([1, 2, 8]), prefix,
                       max(0, own_hi // rng.choice([1, 4, 100])), own_hi, max(1, new // rng.choice([1, 2, 8])), new, heads, cache,
                       rng.random() < 0.5, page, s)
    if op == "fork":
        n = _log(rng, 1, 200)
        ctx = max(1, min(30000, _log(rng, 40, 400000) // n))
        kids, grow = _log(rng, 1, 12), rng.choice([1, 1, _log(rng, 2, 200)])
        return _fork("", n, max(1, kids // 3), kids, ctx // rng.choice([1, 3, 30]), ctx, max(1, grow // rng.choice([1, 3])), grow, heads[1:], cache,
                     page, rng.choice([0.99, 1.05, 1.5, 3.0]), s)
    if op == "compact":
        n = _log(rng, 1, 400)
        ctx = max(20, min(20000, _log(rng, 200, 600000) // n))
        return _compact("", n, ctx // rng.choice([1, 4, 40]), ctx, heads[1:], rng.choice([0.1, 0.3, 0.5, 0.8, 0.97]), cache, page, s)
    n, new = _log(rng, 1, 300), rng.choice([1, _log(rng, 2, 12), _log(rng, 2, 64)])
    vocab = rng.choice([32000, 50257, 128256, 151936, _log(rng, 200, 160000)])
    return _verify("", n, max(1, new // rng.choice([1, 2, 4])), new, vocab, rng.choice(["bf16", "bf16", "f32"]), rng.random() < 0.6, rng.random() < 0.5,
                   rng.choice([0.0, 0.0, 0.3]), s)


def _plain_bytes(case):
    """About what the plain form's intermediate results take."""
    if case["op"] == "shared":
        _, _, ctx, new = _lengths(case)
        longest, T = int((ctx + new).max()), int(new.max())
        return 4 * len(ctx) * longest * (4 * case["Hkv"] * case["d"] + 4 * T * case["Hq"])
    if case["op"] == "verify":
        return 40 * int(_tree(case)[0][-1]) * case["vocab"]
    return 0


def _cost(case):
    w = work(case)
    return w["bytes"] / 5e12 + w["flops"] / 6e14


def draw(rng):
    while True:
        c = _draw_once(rng)
        c.pop("name", None)
        if _cost(c) <= 0.15e-3 and _plain_bytes(c) <= 24 << 30:      # under the largest listed case
            return c


# ---------------------------------------------------------------------------------------------
# structure of a case (lengths, pages, trees): the same for every seed
# ---------------------------------------------------------------------------------------------

def _rng(case, part):
    return np.random.default_rng([case["structure"], part])


def _lengths(case):
    """shared: (first request of every family and the end, prefix of every family, context and new tokens of every request)."""
    rng = _rng(case, 1)
    members = rng.integers(case["members_lo"], case["members_hi"] + 1, case["families"])
    start = np.concatenate([[0], np.cumsum(members)])
    prefix = rng.integers(case["prefix_lo"], case["prefix_hi"] + 1, case["families"])
    n = int(start[-1])
    ctx = np.repeat(prefix, members) + rng.integers(case["own_lo"], case["own_hi"] + 1, n)
    return start, prefix, ctx, rng.integers(case["new_lo"], case["new_hi"] + 1, n)


def _shared_tables(case):
    """(block table, blocks of the pool): whole pages of a family's prefix stand in the tables of all its requests."""
    start, prefix, ctx, new = _lengths(case)
    page = case["page"]
    family = np.repeat(np.arange(case["families"]), np.diff(start))
    whole, pages = prefix // page, (ctx + new + page - 1) // page
    total = int(whole.sum() + (pages - whole[family]).sum())
    pool = int(total * 1.1) + 2
    perm = _rng(case, 2).permutation(pool)
    table = np.zeros((len(ctx), max(1, int(pages.max()))), np.int32)
    at = 0
    first = []
    for w in whole:
        first.append(perm[at:at + w])
        at += w
    for i, p in enumerate(pages):
        w = whole[family[i]]
        table[i, :w] = first[family[i]]
        table[i, w:p] = perm[at:at + p - w]
        at += p - w
    return table, pool


def _pages(case):
    """fork and compact: (lengths, pages of every request, block table, blocks of the pool, holders of every block)."""
    rng = _rng(case, 3)
    n, page = case["n"], case["page"]
    lens = rng.integers(case["ctx_lo"], case["ctx_hi"] + 1, n)
    pages = (lens + page - 1) // page
    total = int(pages.sum())
    if case["op"] == "compact":
        pool, more = max(1, int(math.ceil(total / case["used"]))), 0
    else:
        _, kids, grow = _children(case)
        more = int((((np.repeat(lens, kids) + grow + page - 1) // page - np.repeat(lens // page, kids))).sum())
        pool = max(total, int((total + more) * case["spare"])) + 2
    perm = rng.permutation(pool)
    table = np.zeros((n, int(pages.max()) + (0 if case["op"] == "compact" else case["grow_hi"] // page + 2)), np.int32)
    at = 0
    refs = np.zeros(pool, np.int32)
    for i, p in enumerate(pages):
        table[i, :p] = perm[at:at + p]
        at += p
    refs[perm[:at]] = 1
    return lens, pages, table, pool, refs


def _children(case):
    """fork: (request that every new one comes from, children of every request, tokens that every new one grows by)."""
    rng = _rng(case, 4)
    kids = rng.integers(case["kids_lo"], case["kids_hi"] + 1, case["n"])
    return np.repeat(np.arange(case["n"]), kids), kids, rng.integers(case["grow_lo"], case["grow_hi"] + 1, int(kids.sum()))


def _tree(case):
    """(first token of every request and the end, parent of every token or -1, ancestor bits with its own, number among its siblings)."""
    rng = _rng(case, 5)
    if case["op"] == "verify":
        new = rng.integers(case["new_lo"], case["new_hi"] + 1, case["n"])
        chain = not case["tree"]
    else:
        new, chain = _lengths(case)[3], case["chain"]
    parents, bits, rank = [], [], []
    for T in new:
        par, word, kids = [], [], []
        for t in range(T):
            free = [x for x in range(t) if kids[x] < 4]
            p = t - 1 if chain or t == 0 else free[int(rng.integers(0, len(free)))] if rng.random() < 0.6 else free[-1]
            rank.append(kids[p] if t else 0)
            if t:
                kids[p] += 1
            par.append(p)
            kids.append(0)
            word.append((1 << t) | (word[p] if p >= 0 else 0))
        parents += par
        bits += word
    as_int64 = np.array([b - (1 << 64) if b >> 63 else b for b in bits], np.int64)
    return np.concatenate([[0], np.cumsum(new)]), np.array(parents, np.int64), as_int64, np.array(rank, np.int64)


# ---------------------------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------------------------

def _type(name):
    return {"bf16": torch.bfloat16, "f32": torch.float32}[name]


def _quantize(x):
    """(codes, exponents + 127) as bytes; rows are the last axis."""
    largest = x.abs().amax(-1)
    m, e = torch.frexp(largest)                                    # largest = m 2^e, 448 = 0.875 * 2^9
    E = torch.where(largest > 0, e - 9 + (m > 0.875).to(e.dtype), torch.full_like(e, -126)).clamp(-126, 127)
    factor = ((127 - E) << 23).to(torch.int32).view(torch.float32)     # 2^-E from its bits
    return (x * factor[..., None]).to(torch.float8_e4m3fn).view(torch.uint8), (E + 127).to(torch.uint8)


def _pool(case, gen, blocks):
    Hkv, d, page = case["Hkv"], case["d"], case["page"]

    def rows(outlier):                                             # N(0, 1); some channels of every head larger, as keys have them
        x = torch.randn(blocks, Hkv, page, d, generator=gen, device=DEV)
        return x.mul_(1 + outlier * (torch.rand(1, Hkv, 1, d, generator=gen, device=DEV) < 0.03)) if outlier else x

    by_four = lambda x: x.reshape(blocks, Hkv, page // 4, 4, d).transpose(-1, -2).contiguous()  # noqa: E731
    if case["cache"] == "bf16":
        return rows(4.0).to(torch.bfloat16), by_four(rows(0.0).to(torch.bfloat16)), None
    kc, ks = _quantize(rows(4.0))
    vc, vs = _quantize(rows(0.0))
    scales = torch.stack([ks, vs], dim=2).contiguous().view(torch.float8_e8m0fnu)
    return kc.view(torch.float8_e4m3fn), by_four(vc).view(torch.float8_e4m3fn), scales


def prepare(case, seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(int(seed))
    dev = lambda x, t=torch.int32: torch.from_numpy(np.ascontiguousarray(x)).to(DEV, t)  # noqa: E731
    full = lambda *shape, value=0: torch.full(shape, value, dtype=torch.int32, device=DEV)  # noqa: E731
    s = dict(case=case, op=case["op"])
    if case["op"] == "shared":
        start, _, ctx, new = _lengths(case)
        table, blocks = _shared_tables(case)
        q_start, _, bits, _ = _tree(case)
        s["pool"], s["page"] = _pool(case, gen, blocks), case["page"]
        s["block_table"], s["lens"], s["family_start"], s["q_start"] = dev(table), dev(ctx + new), dev(start), dev(q_start)
        s["longest"], s["max_q"], total = int((ctx + new).max()), int(new.max()), int(new.sum())
        s["row_req"], s["row_t"] = (dev(x, torch.int64) for x in (np.repeat(np.arange(len(new)), new), np.concatenate([np.arange(x) for x in new])))
        s["bits"] = dev(bits, torch.int64)
        s["mask"] = None if case["chain"] else s["bits"]
        s["q"] = torch.randn(total, case["Hq"], case["d"], generator=gen, device=DEV).to(torch.bfloat16)
        s["out"] = torch.empty_like(s["q"])
        s["scale"] = 1.0 / math.sqrt(case["d"])
    elif case["op"] in ("fork", "compact"):
        lens, pages, table, blocks, refs = _pages(case)
        s["pool"], s["page"] = _pool(case, gen, blocks), case["page"]
        s["block_table"], s["lens"], s["pages"], s["refs"] = dev(table), dev(lens), dev(pages), dev(refs)
        if case["op"] == "fork":
            parent, kids, grow = _children(case)
            m = len(parent)
            s["parent"], s["grow"], s["last_kid"] = dev(parent), dev(grow), dev(np.cumsum(kids) - 1)
            s["new"] = full(m, table.shape[1]), full(m), full(m)                       # block table, lengths, pages
            s["back"] = torch.zeros_like(s["block_table"]), torch.empty_like(s["lens"]), torch.empty_like(s["pages"])
            s["served"], s["copy_src"], s["copy_dst"] = full(m), full(m), full(m)
        else:
            moves = blocks // 2 + 1
            s["new_table"], s["new_refs"] = torch.zeros_like(s["block_table"]), torch.empty_like(s["refs"])
            s["copy_src"], s["copy_dst"] = full(moves), full(moves)
    else:
        q_start, parents, bits, rank = _tree(case)
        V, total, n = case["vocab"], len(parents), case["n"]
        first = np.repeat(q_start[:-1], np.diff(q_start))
        s["q_start"], s["bits"], s["max_q"] = dev(q_start), dev(bits, torch.int64), int(np.diff(q_start).max())
        s["mask"] = s["bits"] if case["tree"] else None
        # row of every token's parent (its own for the first one), tokens by number among their siblings (the first ones left out)
        s["parent_row"], s["row_req"] = dev(first + np.maximum(parents, 0), torch.int64), dev(np.repeat(np.arange(n), np.diff(q_start)), torch.int64)
        s["by_rank"] = [dev(np.nonzero((rank == r) & (parents >= 0))[0], torch.int64) for r in range(int(rank.max()) + 1)]
        s["number"] = dev(np.arange(total) - first, torch.int64)
        noise = lambda: -torch.log(-torch.log(torch.rand(total, V, generator=gen, device=DEV).clamp_(1e-20, 1 - 1e-7)))  # noqa: E731
        # logits with a few likely tokens; the draft's are near the target's, and drafted tokens are drawn from them
        target = 2.5 * torch.randn(total, V, generator=gen, device=DEV)
        target.mul_((1 + 0.8 * torch.rand(total, 1, generator=gen, device=DEV)))
        s["target"] = target.to(_type(case["dtype"]))
        s["temperature"] = 0.5 + 0.7 * torch.rand(n, generator=gen, device=DEV)
        near = target + 0.5 * torch.randn(total, V, generator=gen, device=DEV)
        s["draft"] = near.to(_type(case["dtype"])) if case["draft"] else None
        warm = s["temperature"][s["row_req"]][:, None] if case["draft"] else 0.3
        s["tokens"] = (near.to(_type(case["dtype"])).float()[s["parent_row"]] + warm * noise()).argmax(-1).to(torch.int32)
        s["temperature"][:int(round(case["greedy"] * n))] = 0.0
        s["accept_u"], s["sample_u"] = torch.rand(total, generator=gen, device=DEV), torch.rand(n, generator=gen, device=DEV)
        s["keep"], s["keep_count"], s["next"] = full(n, s["max_q"]), full(n), full(n)
    if own:
        # what a serving program keeps from call to call: the cache, a workspace
        from paper_2602_06072_amd import binding as pk
        s["pk"] = pk
        if "pool" in s:
            s["cache"] = pk.KvCache(*s["pool"])
        if case["op"] == "shared":
            s["ws"] = pk.new_shared_tree_workspace(s["lens"].shape[0], s["max_q"], s["q"].shape[0], case["Hq"], case["Hkv"], case["d"])
        elif case["op"] == "verify":
            s["ws"] = pk.new_verify_workspace(case["n"], s["tokens"].shape[0], case["vocab"])
        else:
            s["ws"] = pk.new_pages_workspace(s["refs"].shape[0])
    return s


# ---------------------------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------------------------

def run(s):
    return (_run_own if own else _run_plain)(s)


def _run_own(s):
    pk, op = s["pk"], s["op"]
    if op == "shared":
        pk.shared_tree_attn(s["cache"], s["q"], s["q_start"], s["max_q"], s["mask"], s["block_table"], s["lens"], s["family_start"], s["out"], s["scale"],
                            s["ws"])
    elif op == "fork":
        table, lens, pages = s["new"]
        pk.kv_pages_select(s["block_table"], s["lens"], s["pages"], s["parent"], table, lens, pages, s["refs"], s["page"])
        pk.kv_pages_reserve(table, lens, pages, s["grow"], s["refs"], s["page"], s["served"], s["copy_src"], s["copy_dst"], s["ws"])
        pk.kv_cache_copy(s["cache"], s["copy_src"], s["copy_dst"])
        pk.kv_pages_select(table, lens, pages, s["last_kid"], *s["back"], s["refs"], s["page"])
    elif op == "compact":
        pk.kv_pages_compact(s["block_table"], s["pages"], s["refs"], s["new_table"], s["new_refs"], s["copy_src"], s["copy_dst"], s["ws"])
        pk.kv_cache_copy(s["cache"], s["copy_src"], s["copy_dst"])
    else:
        pk.draft_verify(s["target"], s["draft"], s["tokens"], s["q_start"], s["max_q"], s["mask"], s["temperature"], s["accept_u"], s["sample_u"],
                        s["keep"], s["keep_count"], s["next"], s["ws"])
    return _outputs(s)


def _outputs(s):
    op = s["op"]
    if op == "shared":
        return s["out"]
    if op == "verify":
        return {"keep": s["keep"], "count": s["keep_count"], "next": s["next"]}
    k, v, scales = s["pool"]
    cache = {"k": k, "v": v, "src": s["copy_src"], "dst": s["copy_dst"], **({} if scales is None else {"scales": scales})}
    if op == "compact":
        return {**cache, "table": s["new_table"], "refs": s["new_refs"]}
    return {**cache, "table": s["new"][0], "lens": s["new"][1], "pages": s["new"][2], "served": s["served"], "refs": s["refs"],
            "back": list(s["back"])}


# ------------------------------------------------------------------ the plain form

def _take(pool, slots, page):
    """Rows (f32, [...][Hkv][d]) of slots [...]."""
    blk, off = slots // page, slots % page
    kp, vp, scales = pool
    if scales is None:
        return kp[blk, :, off].float(), vp[blk, :, off // 4, :, off % 4].float()
    k = kp.view(torch.uint8)[blk, :, off].view(torch.float8_e4m3fn).float()
    v = vp.view(torch.uint8)[blk, :, off // 4, :, off % 4].view(torch.float8_e4m3fn).float()
    ks, vs = (scales.view(torch.uint8)[blk, :, i, off].view(torch.float8_e8m0fnu).float()[..., None] for i in (0, 1))
    return k.mul_(ks), v.mul_(vs)


def _attend(s):
    """Keys and values of all requests side by side, padded to the longest."""
    lens, page, n, q = s["lens"].long(), s["page"], s["lens"].shape[0], s["q"].float()
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
    return o.permute(0, 2, 1, 3, 4).reshape(n, T, Hq, d)[s["row_req"], s["row_t"]].to(torch.bfloat16)


def _count(refs, table, pages, by):
    """Adds `by` to the count of every block that a request holds."""
    held = torch.arange(table.shape[1], device=DEV) < pages[:, None]
    refs += torch.zeros_like(refs).index_add_(0, table[held].long(), torch.full_like(table[held], by))


def _select(table, lens, pages, parent, out, refs, page):
    parent = parent.long()
    new_lens = lens[parent]
    new_pages = (new_lens + page - 1) // page
    held = torch.arange(table.shape[1], device=DEV) < new_pages[:, None]
    _count(refs, out[0].copy_(torch.where(held, table[parent], out[0])), new_pages, 1)
    _count(refs, table, pages, -1)
    out[1].copy_(new_lens)
    out[2].copy_(new_pages)


def _reserve(s):
    (table, lens, pages), refs, page = s["new"], s["refs"], s["page"]
    n, most = table.shape
    row, end = torch.arange(n, device=DEV), torch.minimum((lens + s["grow"] + page - 1) // page, torch.full_like(lens, most))
    at = lens // page                                              # page that the next token goes to
    partial = (s["grow"] > 0) & (lens % page > 0) & (pages > at)
    block = table[row, at.clamp(max=most - 1).long()].long()
    shared = partial & (refs[block] > 1)
    # of as many writers as there are holders the last one keeps the page
    writers = torch.zeros_like(refs).index_add_(0, block, shared.to(torch.int32))
    last = torch.full_like(refs, -1).scatter_reduce_(0, block, torch.where(shared, row, -1).to(torch.int32), "amax")
    keeps = shared & (writers[block] == refs[block]) & (last[block] == row)
    copies = shared & ~keeps
    need = (end - pages).clamp(min=0) * (s["grow"] > 0) + copies
    upto = need.cumsum(0)
    free = torch.sort((refs != 0).to(torch.int8), stable=True).indices.to(torch.int32)
    served = (upto <= (refs == 0).sum()) | ((need == 0) & ~keeps)
    need, copies = need * served, copies & served
    begin = upto - need
    # the copy comes first, then the pages behind those that are held
    j = torch.arange(most, device=DEV)
    fresh = (j >= pages[:, None]) & (j < end[:, None]) & (served & (need > 0))[:, None]
    number = begin[:, None] + copies[:, None] + j - pages[:, None]
    s["copy_src"].copy_(torch.where(copies, block, -1))
    s["copy_dst"].copy_(torch.where(copies, free[begin.clamp(max=free.shape[0] - 1)], -1))
    table.copy_(torch.where(fresh, free[number.clamp(0, free.shape[0] - 1)], table))
    here = copies[:, None] & (j == at[:, None])
    table.copy_(torch.where(here, s["copy_dst"][:, None], table))
    refs.index_add_(0, block, -copies.to(torch.int32))
    refs += torch.zeros_like(refs).index_add_(0, table[fresh | here].long(), torch.ones_like(table[fresh | here]))
    pages.copy_(torch.where(served & (need > 0), torch.maximum(pages, end), pages))
    s["served"].copy_(served)


def _copy_pages(s):
    move = s["copy_src"] >= 0
    src, dst = s["copy_src"][move].long(), s["copy_dst"][move].long()
    for x in s["pool"]:
        if x is not None:
            x = x.view(torch.uint8) if x.element_size() == 1 else x
            x[dst] = x[src]


def _compaction(s):
    refs, table = s["refs"], s["block_table"]
    blocks, moves = refs.shape[0], s["copy_src"].shape[0]
    used, number = refs > 0, torch.arange(refs.shape[0], device=DEV)
    in_front = number < used.sum()
    order = lambda x: torch.sort((~x).to(torch.int8), stable=True).indices[:moves]  # noqa: E731
    src, dst = order(used & ~in_front), order(~used & in_front)
    there = torch.arange(src.shape[0], device=DEV) < (used & ~in_front).sum()
    s["copy_src"].fill_(-1)[:src.shape[0]].copy_(torch.where(there, src, -1))
    s["copy_dst"].fill_(-1)[:src.shape[0]].copy_(torch.where(there, dst, -1))
    to = number.clone()
    to[src[there]] = dst[there]
    s["new_refs"].copy_(refs)
    s["new_refs"][dst[there]] = refs[src[there]]
    s["new_refs"][src[there]] = 0
    held = torch.arange(table.shape[1], device=DEV) < s["pages"][:, None]
    s["new_table"].copy_(torch.where(held, to[table.long().clamp(0, blocks - 1)].to(torch.int32), s["new_table"]))


def _weights(logits, warm):
    """Probabilities of rows of logits, in 64 bits."""
    x = logits.double()
    x = torch.where(x.isnan(), -math.inf, x).clamp(max=torch.finfo(torch.float32).max)
    top = x.amax(-1, keepdim=True)
    w = torch.where(x == -math.inf, 0.0, torch.exp((x - top) / warm[:, None]))
    return w / w.sum(-1, keepdim=True).clamp(min=1e-300)


def _judge(s):
    total, V = s["target"].shape
    n = s["q_start"].shape[0] - 1
    req, parent, tokens = s["row_req"], s["parent_row"], s["tokens"].long()
    greedy = ~(s["temperature"] > 0)
    warm = torch.where(greedy, 1.0, s["temperature"]).double()
    P = _weights(s["target"], warm[req])
    top = s["target"].float().amax(-1, keepdim=True)
    best = torch.where(s["target"].float() == top, torch.arange(V, device=DEV), V).amin(-1)
    Q = None if s["draft"] is None else _weights(s["draft"], warm[req])
    # at every token, for its children: what has left P so far, what is left, whether one has stayed
    c, Z = torch.zeros(total, dtype=torch.float64, device=DEV), torch.ones(total, dtype=torch.float64, device=DEV)
    left = P.clone() if Q is None else P
    settled, stays = torch.zeros(total, dtype=torch.bool, device=DEV), s["number"] == 0
    for t in s["by_rank"]:                                         # the first children of all tokens, then the second ones, ...
        p, x, u = parent[t], tokens[t], s["accept_u"][t].double()
        ok = left[p, x] > u * Z[p] if Q is None else P[p, x] > (c[p] + u * Z[p]) * Q[p, x]
        ok = torch.where(greedy[req[t]], best[p] == x, ok) & ~settled[p]
        refused = ~ok & ~settled[p]
        stays[t] = ok
        settled[p] |= ok
        if Q is None:
            Z[p] -= refused * left[p, x]
            left[p, x] *= ~refused
        else:
            r = p[refused]
            c[r] += Z[r]
            Z[r] = (P[r] - c[r][:, None] * Q[r]).clamp_(min=0).sum(-1)
    # a token is kept whose ancestors all stay
    word = torch.zeros(n, dtype=torch.int64, device=DEV).index_add_(0, req, stays.long() << s["number"])
    kept = (s["bits"] & ~word[req]) == 0
    count = torch.zeros(n, dtype=torch.int64, device=DEV).index_add_(0, req, kept.long())
    place = kept.long().cumsum(0) - 1 - (count.cumsum(0) - count)[req]
    keep = torch.full_like(s["keep"], -1)
    keep[req[kept], place[kept]] = s["number"][kept].to(torch.int32)
    last = s["q_start"][:-1].long() + keep.gather(1, count[:, None] - 1)[:, 0]
    # what is left of the last kept token's row
    w = left[last] if Q is None else (P[last] - c[last][:, None] * Q[last]).clamp_(min=0)
    w = torch.where(w.sum(-1, keepdim=True) > 0, w, P[last])
    upto = w.cumsum(-1)
    number = torch.arange(V, device=DEV)
    draw = torch.where((upto > s["sample_u"].double()[:, None] * upto[:, -1:]) & (w > 0), number, V).amin(-1)
    s["next"].copy_(torch.where(greedy, best[last], torch.where(draw < V, draw, torch.where(w > 0, number, -1).amax(-1))))
    s["keep"].copy_(keep)
    s["keep_count"].copy_(count)


def _run_plain(s):
    op = s["op"]
    if op == "shared":
        s["out"] = _attend(s)
    elif op == "fork":
        _select(s["block_table"], s["lens"], s["pages"], s["parent"], s["new"], s["refs"], s["page"])
        _reserve(s)
        _copy_pages(s)
        _select(*s["new"], s["last_kid"], s["back"], s["refs"], s["page"])
    elif op == "compact":
        _compaction(s)
        _copy_pages(s)
    else:
        _judge(s)
    return _outputs(s)


# ---------------------------------------------------------------------------------------------
# what a pass cannot do without
# ---------------------------------------------------------------------------------------------

def _block_bytes(case):
    return 2 * case["Hkv"] * case["page"] * (case["d"] + 1 if case["cache"] == "f8" else 2 * case["d"])


def work(case):
    size = {"bf16": 2, "f32": 4, "f8": 1}
    if case["op"] == "shared":
        start, prefix, ctx, new = _lengths(case)
        page, Hq, Hkv, d = case["page"], case["Hq"], case["Hkv"], case["d"]
        shared = (prefix // page * page) * (np.diff(start) - 1)                     # tokens that are there once and not for each member
        total, fresh = int((ctx + new).sum() - shared.sum()), int(new.sum())
        row = 2 * Hkv * (d * size[case["cache"]] + (1 if case["cache"] == "f8" else 0))
        bits = _tree(case)[2]
        pairs = int((ctx * new).sum()) + sum(bin(int(b) & 0xFFFFFFFFFFFFFFFF).count("1") for b in bits)
        return {"bytes": total * row + 2 * fresh * Hq * d * 2 + 8 * fresh + 4 * int((ctx + new).sum()) // page, "flops": 4 * d * Hq * pairs}
    if case["op"] == "fork":
        lens, pages, table, blocks, refs = _pages(case)
        parent, kids, grow = _children(case)
        page = case["page"]
        copies = int(((kids - 1) * (lens % page > 0)).sum())
        end = (np.repeat(lens, kids) + grow + page - 1) // page
        entries = int(2 * pages.sum() + np.repeat(pages, kids).sum() + end.sum())   # tables in, out, grown, and back
        return {"bytes": 2 * copies * _block_bytes(case) + 4 * entries + 8 * blocks, "flops": entries}
    if case["op"] == "compact":
        lens, pages, table, blocks, refs = _pages(case)
        moves = int((refs[int(pages.sum()):] > 0).sum())
        return {"bytes": 2 * moves * _block_bytes(case) + 8 * int(pages.sum()) + 8 * blocks, "flops": blocks}
    q_start, parents, _, _ = _tree(case)
    first = np.repeat(q_start[:-1], np.diff(q_start))
    inner = len(np.unique((first + parents)[parents >= 0]))                         # tokens with children
    alone = int((np.diff(q_start) == 1).sum())
    rows = inner * (2 if case["draft"] else 1) + alone
    return {"bytes": rows * case["vocab"] * size[case["dtype"]] + 16 * len(parents) + 16 * case["n"], "flops": 4 * rows * case["vocab"]}


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


def _exact_shared(case, s):
    byte_value, page, Hkv, d = _value_of_byte(), case["page"], case["Hkv"], case["d"]
    kp, vp, sc = s["pool"]
    if 30 * kp.numel() > 120e9:
        return None
    look = (lambda x: byte_value[x.view(torch.uint8).long()]) if case["cache"] == "f8" else (lambda x: x.double())
    _, _, ctx, new = _lengths(case)
    table, at, r = s["block_table"].long(), 0, case["Hq"] // case["Hkv"]
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device=DEV)
    for i in range(len(ctx)):
        c, T = int(ctx[i]), int(new[i])
        blocks = table[i, :(c + T + page - 1) // page]
        ki = look(kp[blocks]).transpose(0, 1).reshape(Hkv, -1, d)                   # [Hkv][L][d]
        vi = look(vp[blocks]).permute(1, 0, 2, 4, 3).reshape(Hkv, -1, d)
        if sc is not None:
            e = sc[blocks].view(torch.uint8).double().sub(127).exp2().transpose(0, 1)               # [Hkv][blocks][2][page]
            ki, vi = ki * e[:, :, 0].reshape(Hkv, -1, 1), vi * e[:, :, 1].reshape(Hkv, -1, 1)
        ki, vi = ki[:, :c + T].contiguous(), vi[:, :c + T].contiguous()
        seen = torch.ones(T, c + T, dtype=torch.bool, device=DEV)
        for j in range(T):
            seen[:, c + j] = s["bits"][at:at + T] >> j & 1 != 0
        x = s["q"][at:at + T].double().reshape(T, Hkv, r, d).permute(1, 0, 2, 3).reshape(Hkv, T * r, d).contiguous()
        w = torch.bmm(x, ki.transpose(1, 2).contiguous()) * s["scale"]
        w = w.view(Hkv, T, r, -1).masked_fill(~seen[None, :, None], -math.inf).softmax(-1).view(Hkv, T * r, -1)
        out[at:at + T] = torch.bmm(w, vi).view(Hkv, T, r, d).permute(1, 0, 2, 3).reshape(T, Hkv * r, d)
        at += T
    return out


def _exact_pages(case, s):
    """Page by page on the host."""
    lens, pages, table, blocks, refs = _pages(case)
    page, refs = case["page"], refs.copy()
    if case["op"] == "compact":
        used = int((refs > 0).sum())
        moves = len(s["copy_src"])
        src, dst = [b for b in range(used, blocks) if refs[b]][:moves], [b for b in range(used) if not refs[b]][:moves]
        to = dict(zip(src, dst))
        new_table = np.zeros_like(table)
        for i, p in enumerate(pages):
            new_table[i, :p] = [to.get(b, b) for b in table[i, :p]]
        new_refs = refs.copy()
        for a, b in to.items():
            new_refs[b], new_refs[a] = refs[a], 0
        pad = [-1] * (moves - len(src))
        res = {"src": src + pad, "dst": dst[:len(src)] + pad, "table": new_table, "refs": new_refs}
        moved = list(to.items())
    else:
        parent, kids, grow = _children(case)
        m = len(parent)
        new_table, new_pages = np.zeros((m, table.shape[1]), np.int32), pages[parent].copy()
        for i, p in enumerate(parent):
            new_table[i, :pages[p]] = table[p, :pages[p]]
            refs[table[p, :pages[p]]] += 1
        for j, p in enumerate(pages):
            refs[table[j, :p]] -= 1
        held_by, src, dst, served = refs.copy(), [-1] * m, [-1] * m, [0] * m
        writes = lambda i: grow[i] > 0 and lens[parent[i]] % page > 0  # noqa: E731
        writers = {}
        for i in range(m):
            if writes(i):
                writers.setdefault(int(new_table[i, lens[parent[i]] // page]), []).append(i)
        keeper = {w[-1] for b, w in writers.items() if held_by[b] > 1 and len(w) == held_by[b]}
        free = [b for b in range(blocks) if refs[b] == 0]
        used, short = 0, False
        for i in range(m):
            length = int(lens[parent[i]])
            at = length // page
            end = min(-(-(length + int(grow[i])) // page), table.shape[1])
            copy = writes(i) and held_by[new_table[i, at]] > 1 and i not in keeper
            need = (max(0, end - int(new_pages[i])) if grow[i] else 0) + int(copy)
            short = short or used + need > len(free)
            if short and (need or i in keeper):
                continue
            served[i] = 1
            got = free[used:used + need]
            used += need
            if copy:
                src[i], dst[i] = int(new_table[i, at]), got.pop(0)
                refs[src[i]] -= 1
                new_table[i, at] = dst[i]
                refs[dst[i]] += 1
            for b in got:
                new_table[i, new_pages[i]] = b
                new_pages[i] += 1
                refs[b] += 1
        back_table, back_pages, last = np.zeros_like(table), (lens + page - 1) // page, np.cumsum(kids) - 1
        held = refs * 0
        for j in range(len(lens)):
            back_table[j, :back_pages[j]] = new_table[last[j], :back_pages[j]]
            held[back_table[j, :back_pages[j]]] += 1
        res = {"src": src, "dst": dst, "table": new_table, "lens": lens[parent], "pages": new_pages, "served": served, "refs": held,
               "back": [back_table, lens, back_pages]}
        moved = [(a, b) for a, b in zip(src, dst) if a >= 0]
    whole = lambda v: [whole(x) for x in v] if isinstance(v, list) and v and isinstance(v[0], np.ndarray) else torch.from_numpy(np.array(v, np.int32))  # noqa: E731
    res = {k: whole(v) for k, v in res.items()}
    k, v, sc = (None if x is None else x.clone() for x in s["pool"])
    for x in (k, v, sc):
        if x is not None and moved:
            y = x.view(torch.uint8) if x.element_size() == 1 else x
            a, b = (torch.tensor(z, device=DEV) for z in zip(*moved))
            y[b] = y[a]
    return {**res, "k": k, "v": v, **({} if sc is None else {"scales": sc})}


def _exact_verify(case, s):
    """Request by request, token by token."""
    q_start, parents, _, _ = _tree(case)
    if len(parents) * case["vocab"] > 2e8:
        return None
    keep = np.full((case["n"], s["max_q"]), -1, np.int32)
    count, after = np.zeros(case["n"], np.int32), np.zeros(case["n"], np.int32)
    tokens, accept, sample, warm = (s[x].double().cpu().numpy() for x in ("tokens", "accept_u", "sample_u", "temperature"))

    def probabilities(logits, i):
        x = logits.double()
        return torch.softmax(x / warm[i], -1)

    for i in range(case["n"]):
        a, T = int(q_start[i]), int(q_start[i + 1] - q_start[i])
        at, path, row = 0, [0], None
        for t in range(1, T):
            if parents[a + t] != at:
                continue
            x = int(tokens[a + t])
            logits = s["target"][a + at].float()
            if warm[i] <= 0:
                if int(torch.nonzero(logits == logits.max())[0]) == x:
                    at, row = t, None
                    path.append(t)
                continue
            if row is None:
                row = probabilities(logits, i)                     # what is left, normalised
                other = None if s["draft"] is None else probabilities(s["draft"][a + at].float(), i)
            p = float(row[x])
            if p > accept[a + t] * (1.0 if other is None else float(other[x])):
                at, row = t, None
                path.append(t)
                continue
            if other is None:
                row = row.clone()
                row[x] = 0.0
            else:
                row = (row - other).clamp(min=0)
            row = row / row.sum()
        logits = s["target"][a + at].float()
        if warm[i] <= 0:
            after[i] = int(torch.nonzero(logits == logits.max())[0])
        else:
            row = probabilities(logits, i) if row is None else row
            upto = row.cumsum(0)
            after[i] = int(torch.nonzero((upto > sample[i] * upto[-1]) & (row > 0))[0])
        keep[i, :len(path)] = path
        count[i] = len(path)
    return {"keep": torch.from_numpy(keep), "count": torch.from_numpy(count), "next": torch.from_numpy(after)}


def exact(case, seed):
    s = prepare(case, seed)
    return {"shared": _exact_shared, "verify": _exact_verify}.get(case["op"], _exact_pages)(case, s)
