"""Norm and rotation, the paged cache and the attention of drafted tokens through the public calls, against the
definitions in 64 bits (oracle/cache.py).

Tolerances.  fp32 results of norm and rotation: a sum of d squares, a square root and four products, at most
(d / 8 + 16) roundings of 2^-24 of the pair's magnitude: 3e-6.  bf16: half a unit in the last place (2^-8 of the
value) more.  Codes of rows that are not normed have to be equal; normed rows may fall on the other side of a tie: half
a step of the format (2^-4 of the value, 2^-10 of the scale below the normal numbers), a tenth of a percent for the
fp32 arithmetic in front.  Attention: probabilities are rounded to bf16 (2^-8 each, above and below the fraction),
scores are fp32 sums (exp of an error of 2e-5): 2^-8 (sum p |v| + |o|) + 1e-4 sum p |v|, and 2^-8 |o| for bf16
output."""
import numpy as np
import pytest
import torch

from oracle import cache as oc
from paper_2602_06072_amd import binding as pk

pytestmark = pytest.mark.gpu
DEV = "cuda"
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
VALUES = oc.e4m3_values()


def gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def randn(g, *shape, dtype=torch.bfloat16):
    return torch.randn(*shape, generator=g, device=DEV).to(dtype)


def f64(x):
    return x.detach().double().cpu().numpy()


def table_of(max_pos, rot):
    freq = 10000.0 ** (-torch.arange(0, rot, 2, dtype=torch.float64) / rot)
    ang = torch.arange(max_pos, dtype=torch.float64)[:, None] * freq
    return torch.stack([ang.cos(), ang.sin()], 1).float().contiguous().to(DEV)


def token_major(cache):
    """(K codes, V codes, scales of K, scales of V), rows by slot, in 64 bits, from the layout that the header describes."""
    raw = lambda x: x.cpu().view(torch.uint8).numpy() if x.element_size() == 1 else x.double().cpu().numpy()  # noqa: E731
    k, v = raw(cache.k), raw(cache.v)
    if cache.dtype == pk.PK_F8:
        k, v = VALUES[k], VALUES[v]
    B, H, P, d = k.shape
    k = k.transpose(0, 2, 1, 3).reshape(B * P, H, d)
    v = v.transpose(0, 2, 4, 1, 3).reshape(B * P, H, d)
    if cache.dtype == pk.PK_BF16:
        return k, v, np.ones((B * P, H)), np.ones((B * P, H))
    s = 2.0 ** (raw(cache.scales).astype(np.float64) - 127)
    s = s.transpose(0, 3, 1, 2).reshape(B * P, H, 2)
    return k, v, s[..., 0], s[..., 1]


def close(got, want, tol):
    assert got.shape == want.shape
    assert np.array_equal(np.isnan(got), np.isnan(want))
    bad = np.abs(np.nan_to_num(got) - np.nan_to_num(want)) > np.nan_to_num(tol) + 1e-30
    assert not bad.any(), (int(bad.sum()), bad.size, float(np.nanmax(np.abs(got - want))))


# ------------------------------------------------------------------ norm and rotation

SHAPES = [(1, 32, 8, 128, 128), (7, 8, 2, 64, 64), (33, 5, 1, 128, 64), (130, 3, 3, 96, 32), (65, 28, 4, 256, 256), (600, 32, 8, 128, 128), (3, 2, 2, 40, 16), (9, 64, 8, 8, 0)]


@pytest.mark.parametrize("tokens, Hq, Hkv, d, rot", SHAPES)
@pytest.mark.parametrize("dtype, out", [("bf16", "bf16"), ("f32", "f32"), ("bf16", "f32"), ("f32", "bf16")])
@pytest.mark.parametrize("axes, interleaved, norm", [(1, False, True), (3, False, False), (3, True, True), (1, True, False)])
def test_norm_and_rotation(tokens, Hq, Hkv, d, rot, dtype, out, axes, interleaved, norm):
    g = gen(tokens + d)
    t = TYPES[dtype]
    qkv = randn(g, tokens, Hq + 2 * Hkv, d, dtype=t) * torch.exp(2 * torch.randn(tokens, Hq + 2 * Hkv, 1, generator=g, device=DEV)).to(t)
    q, k = qkv[:, :Hq], qkv[:, Hq:Hq + Hkv]
    wq, wk = (randn(g, d, dtype=t) if norm else None for _ in "qk")
    rope, table, pos, axis = None, None, None, None
    if rot:
        table, pos = table_of(211, rot), torch.randint(0, 211, (axes, tokens), generator=g, device=DEV, dtype=torch.int32)
        axis = None if axes == 1 else [p % 3 if interleaved else min(2, 3 * p // (rot // 2)) for p in range(rot // 2)]
        rope = pk.Rope(table, pos, axis, interleaved)
    qo, ko = (torch.full((tokens, h, d), 7.0, dtype=TYPES[out], device=DEV) for h in (Hq, Hkv))
    pk.qk_norm_rope(q, k, qo, ko, wq, wk, 1e-5, rope)
    torch.cuda.synchronize()
    for x, w, y in ((q, wq, qo), (k, wk, ko)):
        want = oc.norm_rope(f64(x), None if w is None else f64(w), 1e-5, None if table is None else f64(table), None if pos is None else pos.cpu().numpy(), axis, interleaved)
        top = np.abs(want).max(-1, keepdims=True) if w is None else np.abs(oc.norm_rope(f64(x), f64(w), 1e-5, None, None, None, False)).max(-1, keepdims=True)
        close(f64(y), want, 3e-6 * np.maximum(top, np.abs(want)) + (2.0 ** -8 * np.abs(want) if out == "bf16" else 0))


def test_norm_and_rotation_in_place_strided_and_on_another_stream():
    g = gen(5)
    base = randn(g, 50, 24, 160)                                   # rows wider than d, tokens wider than the heads
    q, k = base[:, :8, :128], base[:, 10:12, :128]
    table, pos = table_of(64, 128), torch.randint(0, 64, (50,), generator=g, device=DEV, dtype=torch.int32)
    want_q, want_k = torch.empty(50, 8, 128, dtype=torch.bfloat16, device=DEV), torch.empty(50, 2, 128, dtype=torch.bfloat16, device=DEV)
    w = randn(g, 128)
    rope = pk.Rope(table, pos)
    pk.qk_norm_rope(q, k, want_q, want_k, w, w, 1e-6, rope)
    before = base.clone()
    heads_first = torch.empty(8, 50, 128, dtype=torch.bfloat16, device=DEV)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    pk.qk_norm_rope(q, k, heads_first.transpose(0, 1), torch.empty_like(want_k), w, w, 1e-6, rope, stream=s)
    s.synchronize()
    assert torch.equal(heads_first.transpose(0, 1), want_q)
    pk.qk_norm_rope(q, k, q, k, w, w, 1e-6, rope)
    assert torch.equal(q, want_q) and torch.equal(k, want_k)
    base[:, :8, :128], base[:, 10:12, :128] = before[:, :8, :128], before[:, 10:12, :128]
    assert torch.equal(base, before)                               # nothing beside the rows was written


def test_rows_of_zeros_infinities_and_positions_outside_of_the_table():
    x = torch.zeros(4, 1, 64, dtype=torch.float32, device=DEV)
    x[1, 0, 3], x[2, 0, 5], x[3] = float("inf"), float("nan"), 1.0
    table = table_of(10, 64)
    out, ko = torch.empty_like(x), torch.empty_like(x)
    w = torch.ones(64, device=DEV)
    pk.qk_norm_rope(x, x, out, ko, w, None, 0.0, None)             # eps 0: a row of zeros has no direction
    assert torch.isnan(out[0]).all() and torch.isnan(out[2]).all() and torch.equal(out[3], x[3])
    assert torch.equal(ko[0], x[0]) and torch.equal(ko[1], x[1]) and torch.isnan(ko[2, 0, 5])
    pos = torch.tensor([-5, 0, 9, 1 << 30], dtype=torch.int32, device=DEV)
    y = torch.ones(4, 1, 64, dtype=torch.float32, device=DEV)
    pk.qk_norm_rope(y, y, out, ko, None, None, 0.0, pk.Rope(table, pos))
    assert torch.equal(out[0], out[1]) and torch.equal(out[2], out[3]) and torch.equal(out[0], y[0])


# ------------------------------------------------------------------ the cache

@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("cache", [pk.PK_F8, pk.PK_BF16])
@pytest.mark.parametrize("tokens, Hkv, d, page", [(1, 8, 128, 16), (37, 2, 64, 48), (300, 5, 128, 32), (64, 1, 64, 16), (515, 8, 128, 16)])
@pytest.mark.parametrize("order", ["rising", "random"])
def test_cache_write(tokens, Hkv, d, page, cache, dtype, order):
    g = gen(tokens)
    blocks = tokens // page + 3
    c = pk.new_kv_cache(blocks, page, Hkv, d, cache)
    for x in (c.k, c.v) + ((c.scales,) if cache == pk.PK_F8 else ()):
        x.view(torch.uint8).fill_(0x5A)
    spread = torch.exp(3 * torch.randn(tokens, Hkv, 1, generator=g, device=DEV))
    k, v = ((torch.randn(tokens, Hkv, d, generator=g, device=DEV) * spread).to(TYPES[dtype]) for _ in "kv")
    k[0, 0] = 0.0
    v[tokens // 2, 0, 3:6] = torch.tensor([float("inf"), -float("inf"), float("nan")], device=DEV).to(v.dtype)
    slots = torch.arange(5, 5 + tokens, device=DEV) if order == "rising" else torch.randperm(blocks * page, generator=g, device=DEV)[:tokens]
    slots = slots.clone()
    if tokens > 4:
        slots[1], slots[3] = -1, blocks * page                     # not written
    old = token_major(c)
    pk.kv_cache_write(c, k, v, slots)
    torch.cuda.synchronize()
    got, at = token_major(c), slots.cpu().numpy()
    ok = (at >= 0) & (at < blocks * page)
    for i, x in enumerate((k, v)):
        want, scale = old[i].copy(), old[2 + i].copy()
        if cache == pk.PK_F8:
            codes, E = oc.quantize(f64(x))
            want[at[ok]], scale[at[ok]] = codes[ok], 2.0 ** E[ok]
        else:
            want[at[ok]] = f64(x.to(torch.bfloat16))[ok]
        assert np.array_equal(got[i], want, equal_nan=True)
        assert np.array_equal(got[2 + i], scale)


@pytest.mark.parametrize("tokens, Hq, Hkv, d", [(1, 32, 8, 128), (20, 8, 8, 64), (333, 7, 1, 128), (90, 40, 8, 64)])
@pytest.mark.parametrize("cache, dtype, norm", [(pk.PK_F8, "bf16", True), (pk.PK_F8, "f32", False), (pk.PK_BF16, "bf16", True)])
def test_norm_rotation_and_cache_write_in_one_launch(tokens, Hq, Hkv, d, cache, dtype, norm):
    g = gen(tokens + Hq)
    page, t = 16, TYPES[dtype]
    c = pk.new_kv_cache(tokens // page + 2, page, Hkv, d, cache)
    qkv = randn(g, tokens, Hq + 2 * Hkv, d, dtype=t)
    q, k, v = qkv[:, :Hq], qkv[:, Hq:Hq + Hkv], qkv[:, Hq + Hkv:]
    wq, wk = (randn(g, d, dtype=t) if norm else None for _ in "qk")
    table, pos = table_of(100, d), torch.randint(0, 100, (tokens,), generator=g, device=DEV, dtype=torch.int32)
    rope = pk.Rope(table, pos)
    slots = torch.randperm(c.num_blocks * page, generator=g, device=DEV)[:tokens]
    qo, ko, q_alone = torch.empty_like(q).contiguous(), torch.empty(tokens, Hkv, d, dtype=torch.float32, device=DEV), torch.empty(tokens, Hq, d, dtype=t, device=DEV)
    pk.qkv_cache_write(c, q, k, v, slots, qo, wq, wk, 1e-6, rope)
    pk.qk_norm_rope(q, k, q_alone, torch.empty(tokens, Hkv, d, dtype=t, device=DEV), wq, wk, 1e-6, rope)
    assert torch.equal(qo, q_alone)
    want = oc.norm_rope(f64(k), None if wk is None else f64(wk), 1e-6, f64(table), pos.cpu().numpy()[None], None, False)
    kc, vc, ks, vs = (x[slots.cpu().numpy()] for x in token_major(c))
    if cache == pk.PK_F8:
        close(kc * ks[..., None], want, 1.001 * np.maximum(2.0 ** -4 * np.abs(want), 2.0 ** -10 * ks[..., None]))
        codes, E = oc.quantize(f64(v))
        assert np.array_equal(vc, codes) and np.array_equal(vs, 2.0 ** E)
        top = np.abs(kc).max(-1)
        assert (top <= 448).all() and (top >= 208).all()           # the scale is the smallest one
    else:
        close(kc, want, 2.0 ** -8 * np.abs(want) + 3e-6 * np.abs(want).max(-1, keepdims=True))
        assert np.array_equal(vc, f64(v.to(torch.bfloat16)))


def random_cache(g, blocks, page, Hkv, d, dtype, spread=1.0):
    c = pk.new_kv_cache(blocks, page, Hkv, d, dtype)
    rows = lambda: torch.randn(blocks * page, Hkv, d, generator=g, device=DEV) * torch.exp(spread * torch.randn(blocks * page, Hkv, 1, generator=g, device=DEV))  # noqa: E731
    pk.kv_cache_write(c, rows(), rows(), torch.arange(blocks * page, device=DEV))
    return c


def placement(rng, lens, page, blocks):
    """Block table with garbage where a request has no pages; slots of every request's tokens."""
    width = max(1, max((int(x) + page - 1) // page for x in lens)) + 1
    table = rng.integers(-(1 << 30), 1 << 30, size=(len(lens), width)).astype(np.int32)
    perm, at, slots = rng.permutation(blocks), 0, []
    for i, x in enumerate(lens):
        b = (int(x) + page - 1) // page
        table[i, :b] = perm[at:at + b]
        at += b
        pos = np.arange(int(x))
        slots.append(table[i, pos // page].astype(np.int64) * page + pos % page)
    assert at <= blocks
    return torch.from_numpy(table).to(DEV), slots


@pytest.mark.parametrize("out", ["bf16", "f32"])
@pytest.mark.parametrize("cache", [pk.PK_F8, pk.PK_BF16])
@pytest.mark.parametrize("lens, Hkv, d, page", [([1], 8, 128, 16), ([0, 17, 16, 0, 15, 300], 2, 64, 16), ([700, 3, 64], 5, 128, 48), ([129, 1, 128], 8, 64, 128)])
def test_cache_read(lens, Hkv, d, page, cache, out):
    g, rng = gen(sum(lens)), np.random.default_rng(len(lens))
    blocks = sum((x + page - 1) // page for x in lens) + 2
    c = random_cache(g, blocks, page, Hkv, d, cache, 3.0)
    table, slots = placement(rng, lens, page, blocks)
    gap = 3                                                        # rows in front of every request that are somebody else's
    start = np.cumsum([gap] + [x + gap for x in lens])[:len(lens)]
    rows = sum(lens) + gap * (len(lens) + 1)
    ko, vo = (torch.full((rows, Hkv, d), 7.0, dtype=TYPES[out], device=DEV) for _ in "kv")
    pk.kv_cache_read(c, table, torch.tensor(lens, dtype=torch.int32, device=DEV), torch.from_numpy(start.astype(np.int32)).to(DEV), ko, vo)
    torch.cuda.synchronize()
    k, v, ks, vs = token_major(c)
    for got, code, scale in ((ko, k, ks), (vo, v, vs)):
        want = np.full((rows, Hkv, d), 7.0)
        for s, at in zip(start, slots):
            want[s:s + len(at)] = code[at] * scale[at][..., None]
        assert np.array_equal(f64(got), want)


def test_cache_read_clamps_lengths_and_rows():
    g, page = gen(8), 16
    c = random_cache(g, 4, page, 2, 64, pk.PK_F8)
    table = torch.arange(4, dtype=torch.int32, device=DEV).view(2, 2)
    ko, vo = (torch.full((40, 2, 64), 7.0, dtype=torch.float32, device=DEV) for _ in "kv")
    lens = torch.tensor([1 << 30, -4], dtype=torch.int32, device=DEV)
    pk.kv_cache_read(c, table, lens, torch.tensor([20, 0], dtype=torch.int32, device=DEV), ko, vo)      # 32 tokens, 20 rows left
    k, _, ks, _ = token_major(c)
    assert np.array_equal(f64(ko[20:]), (k * ks[..., None])[:20]) and (ko[:20] == 7).all()


# ------------------------------------------------------------------ attention of drafted tokens

def make(seed, ctx, drafts, Hq, Hkv, d, page, cache, spread=0.3, hostile=True):
    """Everything a call takes, the cache with NaN wherever no token of a request is."""
    g, rng = gen(seed), np.random.default_rng(seed)
    lens = [a + b for a, b in zip(ctx, drafts)]
    blocks = sum((x + page - 1) // page for x in lens) + 3
    c = random_cache(g, blocks, page, Hkv, d, cache, spread)
    table, slots = placement(rng, lens, page, blocks)
    if hostile:
        used = np.zeros(blocks * page, bool)
        used[np.concatenate(slots)] = True
        free = torch.from_numpy(np.nonzero(~used)[0]).to(DEV)
        nan = torch.full((len(free), Hkv, d), float("nan"), device=DEV)
        pk.kv_cache_write(c, nan, nan, free)
        if cache == pk.PK_F8:
            c.scales.view(torch.uint8).permute(0, 3, 1, 2).reshape(-1, Hkv, 2)      # (a copy: written below by its own indices)
            b, off = free // page, free % page
            c.scales.view(torch.uint8)[b, :, :, off] = 255
    q_start = np.concatenate([[0], np.cumsum(drafts)]).astype(np.int32)
    q = randn(g, int(q_start[-1]), Hq, d)
    return dict(c=c, table=table, slots=slots, lens=lens, drafts=drafts, q_start=q_start, q=q, max_q=max(drafts), scale=d ** -0.5, rng=rng)


def masks(s, kind):
    """None, or words [total]: random bits ("bits": some rows see no drafted token), or trees."""
    if kind == "chain":
        return None
    words = []
    for T in s["drafts"]:
        own = []
        for t in range(T):
            if kind == "bits":
                own.append(int(s["rng"].integers(0, 1 << 63)) * 2 + int(s["rng"].integers(0, 2)) if t % 3 else 0)
            else:
                p = int(s["rng"].integers(-1, t)) if t else -1
                own.append((1 << t) | (own[p] if p >= 0 else 0))
        words += own
    return np.array([w & (2 ** 64 - 1) for w in words], dtype=np.uint64)


def call(s, mask, out_dtype=torch.bfloat16, ws=None, stream=None):
    dev = lambda x: torch.from_numpy(np.ascontiguousarray(x)).to(DEV)  # noqa: E731
    out = torch.full(s["q"].shape, 7.0, dtype=out_dtype, device=DEV)
    c = s["c"]
    if ws is None:
        ws = pk.new_tree_workspace(len(s["lens"]), s["max_q"], s["q"].shape[1], c.Hkv, c.d)
    pk.tree_attn(c, s["q"], dev(s["q_start"]), s["max_q"], None if mask is None else dev(mask.view(np.int64)), s["table"],
                 dev(np.array(s["lens"], np.int32)), out, s["scale"], ws, stream=stream)
    return out


def check(s, mask, out):
    k, v, ks, vs = token_major(s["c"])
    q, got = f64(s["q"]), f64(out)
    for i, at in enumerate(s["slots"]):
        a, b = s["q_start"][i], s["q_start"][i + 1]
        if a == b:
            continue
        with np.errstate(invalid="ignore"):
            want, spread = oc.tree_attention(q[a:b], k[at] * ks[at][..., None], v[at] * vs[at][..., None], int(b - a),
                                             None if mask is None else mask[a:b], s["scale"])
        tol = 2.0 ** -8 * (spread + np.abs(want)) + 1e-4 * spread + (2.0 ** -8 * np.abs(want) if out.dtype == torch.bfloat16 else 0)
        close(got[a:b], want, tol)


HEADS = [(8, 2, 64), (8, 8, 128), (7, 1, 128), (40, 8, 64), (64, 8, 128), (32, 1, 128)]
BATCHES = [([0], [1]), ([1, 31, 32, 33], [1, 1, 1, 1]), ([0, 5, 200, 63], [3, 0, 7, 1]), ([700, 0, 17], [64, 64, 33]), ([2500], [2]), ([15, 1], [17, 16])]


@pytest.mark.parametrize("Hq, Hkv, d", HEADS)
@pytest.mark.parametrize("ctx, drafts", BATCHES)
@pytest.mark.parametrize("kind, cache, page", [("tree", pk.PK_F8, 16), ("chain", pk.PK_F8, 48), ("bits", pk.PK_F8, 16), ("tree", pk.PK_BF16, 32), ("bits", pk.PK_BF16, 16)])
def test_attention_of_drafted_tokens(Hq, Hkv, d, ctx, drafts, kind, cache, page):
    if sum(drafts) * Hq * (max(ctx) + 64) > 3e6:
        Hq, Hkv = Hq // Hkv, 1                                     # (the oracle's time)
    s = make(Hq + sum(ctx), ctx, drafts, Hq, Hkv, d, page, cache)
    mask = masks(s, kind)
    out = call(s, mask, torch.float32 if kind == "bits" else torch.bfloat16)
    torch.cuda.synchronize()
    check(s, mask, out)


def test_rows_that_see_nothing_are_zero():
    s = make(3, [0, 0], [4, 40], 8, 2, 128, 16, pk.PK_F8)
    mask = np.zeros(44, np.uint64)
    mask[2] = 1
    out = call(s, mask)
    assert (out[[0, 1, 3]] == 0).all() and (out[4:] == 0).all() and (out[2] != 0).any()
    check(s, mask, out)


@pytest.mark.parametrize("cache", [pk.PK_F8, pk.PK_BF16])
@pytest.mark.parametrize("drafts", [4, 23])
def test_what_a_row_does_not_see_does_not_reach_it(cache, drafts):
    """A NaN in K or V of one drafted token reaches the rows that see it, in V its own column alone, and no other row."""
    s = make(11, [50], [drafts], 8, 2, 64, 16, cache)
    mask = np.array([1 << t | (1 if t % 2 else 0) for t in range(drafts)], np.uint64)      # odd tokens see token 0 and themselves, even ones themselves
    clean = call(s, mask)
    c, slot = s["c"], torch.tensor([int(s["slots"][0][50]), int(s["slots"][0][52])], device=DEV)
    g = gen(1)
    k, v = torch.randn(2, 2, 64, generator=g, device=DEV), torch.randn(2, 2, 64, generator=g, device=DEV)
    k[1, 0, 3] = float("nan")                                      # token 2, KV head 0: seen by itself alone
    v[0, 1, 5] = float("nan")                                      # token 0, KV head 1, column 5: seen by itself and the odd ones
    pk.kv_cache_write(c, k, v, slot)
    out = call(s, mask)
    check(s, mask, out)
    nan = torch.isnan(out)
    rows = torch.zeros(drafts, dtype=torch.bool, device=DEV)
    rows[0], rows[1::2] = True, True
    assert nan[2, :4].all() and not nan[torch.arange(drafts) != 2, :4].any()
    assert torch.equal(nan[:, 4:, 5], rows[:, None].expand(-1, 4)) and not nan[:, 4:, :5].any() and not nan[:, 4:, 6:].any()
    untouched = ~rows
    untouched[2] = False
    assert torch.equal(out[untouched], clean[untouched])


@pytest.mark.parametrize("spread", [0.0, 4.0])
def test_sharp_and_far_apart_scores(spread):
    s = make(21, [900], [5], 8, 2, 128, 16, pk.PK_F8, spread)
    s["scale"] = 1.0
    mask = masks(s, "tree")
    check(s, mask, call(s, mask))


def test_lengths_shorter_than_the_drafts_are_bounded():
    """A request whose length says less than its drafted tokens: those in front of the first token are not there."""
    s = make(31, [0, 6], [5, 3], 4, 2, 64, 16, pk.PK_F8)
    s["lens"] = [2, 9]
    k, v, ks, vs = token_major(s["c"])
    out = call(s, None)
    # of request 0 tokens 3 and 4 are in slots 0 and 1; token t sees those up to itself
    at = s["slots"][0][:2]
    q = f64(s["q"])
    assert (out[:3] == 0).all()
    for t in (3, 4):
        want, spread = oc.tree_attention(q[t:t + 1], (k[at] * ks[at][..., None])[:t - 2], (v[at] * vs[at][..., None])[:t - 2], 0, None, s["scale"])
        close(f64(out[t:t + 1]), want, 2.0 ** -8 * (spread + 2 * np.abs(want)) + 1e-4 * spread)


def test_results_repeat_and_the_workspace_serves_every_smaller_call():
    big = make(41, [3000, 10, 900], [9, 1, 30], 16, 2, 128, 16, pk.PK_F8)
    small = make(42, [400], [2], 16, 2, 128, 16, pk.PK_F8)
    ws = pk.new_tree_workspace(3, 30, 16, 2, 128)
    mask = masks(big, "tree")
    first = call(big, mask, ws=ws)
    a = call(small, None, ws=ws)
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    again = call(big, mask, ws=ws, stream=stream)
    stream.synchronize()
    assert torch.equal(first, again) and torch.equal(a, call(small, None, ws=ws))
    check(big, mask, first)


def test_a_captured_step_replays_while_lengths_grow():
    s = make(51, [100, 40], [3, 3], 8, 2, 128, 16, pk.PK_F8)
    dev = lambda x: torch.from_numpy(np.ascontiguousarray(x)).to(DEV)  # noqa: E731
    q_start, lens = dev(s["q_start"]), dev(np.array([20, 20], np.int32))
    out = torch.zeros_like(s["q"])
    ws = pk.new_tree_workspace(2, 3, 8, 2, 128)
    args = (s["c"], s["q"], q_start, 3, None, s["table"], lens, out, s["scale"], ws)
    pk.tree_attn(*args)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        pk.tree_attn(*args)
    for now in ([20, 20], [103, 43], [64, 7], [103, 3]):
        lens.copy_(torch.tensor(now, dtype=torch.int32))
        out.fill_(7.0)
        graph.replay()
        torch.cuda.synchronize()
        got = out.clone()
        pk.tree_attn(*args)
        torch.cuda.synchronize()
        assert torch.equal(got, out)
        sub = dict(s, lens=now, slots=[a[:x] for a, x in zip(s["slots"], now)])
        check(sub, None, got)


@pytest.mark.parametrize("cache", [pk.PK_F8, pk.PK_BF16])
def test_blocks_beyond_four_gigabytes(cache):
    """Blocks whose byte offsets need more than 32 bits, and slots near the end of such a cache."""
    Hkv, d, page = 8, 128, 16
    blocks = (1 << 32) // (Hkv * d * page) + 40
    c = pk.new_kv_cache(blocks, page, Hkv, d, cache)
    g = gen(61)
    lens, drafts = [120, 33], [4, 1]
    table = np.array([[blocks - 1 - i for i in range(8)], [blocks - 20 - i for i in range(3)] + [0] * 5], np.int32)
    slots = [table[i, np.arange(x) // page].astype(np.int64) * page + np.arange(x) % page for i, x in enumerate(lens)]
    at = torch.from_numpy(np.concatenate(slots)).to(DEV)
    k, v = randn(g, 153, Hkv, d), randn(g, 153, Hkv, d)
    pk.kv_cache_write(c, k, v, at)
    ko, vo = torch.empty_like(k), torch.empty_like(v)
    dev = lambda x: torch.tensor(x, dtype=torch.int32, device=DEV)  # noqa: E731
    tab = torch.from_numpy(table).to(DEV)
    pk.kv_cache_read(c, tab, dev(lens), dev([0, 120]), ko, vo)
    for got, x in ((ko, k), (vo, v)):
        if cache == pk.PK_F8:
            codes, E = oc.quantize(f64(x))
            assert np.array_equal(f64(got), codes * 2.0 ** E[..., None])
        else:
            assert torch.equal(got, x)
    q, out = randn(g, 5, 16, d), torch.empty(5, 16, d, dtype=torch.bfloat16, device=DEV)
    pk.tree_attn(c, q, dev([0, 4, 5]), 4, None, tab, dev(lens), out, 0.1, pk.new_tree_workspace(2, 4, 16, Hkv, d))
    for i, (a, b, r) in enumerate(((0, 4, 0), (4, 5, 120))):
        want, spread = oc.tree_attention(f64(q[a:b]), f64(ko[r:r + lens[i]]), f64(vo[r:r + lens[i]]), drafts[i], None, 0.1)
        close(f64(out[a:b]), want, 2.0 ** -8 * (spread + 2 * np.abs(want)) + 1e-4 * spread)


# ------------------------------------------------------------------ keeping accepted tokens

@pytest.mark.parametrize("cache", [pk.PK_F8, pk.PK_BF16])
@pytest.mark.parametrize("d, page", [(128, 16), (64, 48)])
def test_accepted_tokens_move_up(cache, d, page):
    ctx, drafts = [0, 15, 30, 7, 100], [64, 5, 17, 0, 9]
    s = make(71, ctx, drafts, 4, 2, d, page, cache, hostile=False)
    keep = np.full((5, 20), -9, np.int32)
    kept = [sorted(s["rng"].permutation(64)[:20].tolist()), [0, 1, 2, 3, 4], [16], [], [2, 3, 99]]      # 99: no such token
    for i, x in enumerate(kept):
        keep[i, :len(x)] = x
    count = np.array([20, 5, 1, 3, 3], np.int32)                  # request 3 has no drafted tokens
    dev = lambda x: torch.from_numpy(np.ascontiguousarray(x)).to(DEV)  # noqa: E731
    before = token_major(s["c"])
    new = torch.full((5,), -1, dtype=torch.int32, device=DEV)
    pk.kv_cache_keep(s["c"], s["table"], dev(np.array(s["lens"], np.int32)), dev(s["q_start"]), dev(keep), dev(count), new)
    torch.cuda.synchronize()
    assert new.tolist() == [20, 20, 31, 7, 103]
    after = token_major(s["c"])
    for a, b in zip(before, after):
        want = a.copy()
        for i, x in enumerate(kept):
            for j, t in enumerate(x):
                if t < drafts[i]:
                    want[s["slots"][i][ctx[i] + j]] = a[s["slots"][i][ctx[i] + t]]
        assert np.array_equal(b, want, equal_nan=True)
