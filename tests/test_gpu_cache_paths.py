"""The paged cache and the attention of drafted tokens where the work is divided differently: hundreds of requests,
requests of one wave, pieces in one round and in several, merges, cells of four values behind ragged contexts.

Tolerances are those of test_gpu_cache_step.py (probabilities rounded to bf16, fp32 scores); codes of written rows and of
normed keys have to be those of the exact value."""
import numpy as np
import pytest
import torch

from oracle import cache as oc
from paper_2602_06072_amd import binding as pk
from tests import test_gpu_cache_step as step

pytestmark = pytest.mark.gpu
DEV = "cuda"


def dense(s, mask, out):
    """step.check with the attention of a request as products in 64 bits."""
    k, v, ks, vs = (torch.from_numpy(x).to(DEV) for x in step.token_major(s["c"]))
    q = s["q"].double()
    T, Hq, d = q.shape
    Hkv = s["c"].Hkv
    for i, at in enumerate(s["slots"]):
        a, b = int(s["q_start"][i]), int(s["q_start"][i + 1])
        if a == b:
            continue
        at = torch.from_numpy(np.asarray(at)).to(DEV)
        L, ctx = len(at), len(at) - (b - a)
        seen = torch.ones(b - a, L, dtype=torch.bool, device=DEV)
        words = [2 ** (t + 1) - 1 for t in range(b - a)] if mask is None else [int(x) for x in mask[a:b]]
        seen[:, ctx:] = torch.tensor([[bool(w >> j & 1) for j in range(b - a)] for w in words], device=DEV)
        for h in range(Hkv):
            heads = slice(h * (Hq // Hkv), (h + 1) * (Hq // Hkv))
            kk, vv = k[at, h] * ks[at, h, None], v[at, h] * vs[at, h, None]
            sc = (s["scale"] * (q[a:b, heads].reshape(-1, d) @ kk.t().contiguous())).view(b - a, -1, L)
            sc = sc.masked_fill(~seen[:, None], -torch.inf)
            p = torch.exp(sc - sc.amax(-1, keepdim=True).clamp(min=-1e300))
            p = (p / p.sum(-1, keepdim=True).clamp(min=1e-300)).view(-1, L)
            want, spread = (p @ x for x in (vv, vv.abs()))
            got = out[a:b, heads].double().reshape(-1, d)
            tol = 2.0 ** -8 * (spread + want.abs()) + 1e-4 * spread + (2.0 ** -8 * want.abs() if out.dtype == torch.bfloat16 else 0)
            off = (got - want).abs() - tol
            assert torch.isfinite(got).all() and float(off.max()) <= 1e-30, (i, h, float(off.max()))


def ragged(seed, n, top, most, none=0.1):
    """n contexts up to `top` (few long ones) and numbers of drafted tokens up to `most`, some requests without any."""
    rng = np.random.default_rng(seed)
    ctx = np.floor((top + 1) * rng.random(n) ** 3).astype(int)
    drafts = rng.integers(1, most + 1, n) * (rng.random(n) >= none)
    drafts[0] = most
    return [int(x) for x in ctx], [int(x) for x in drafts]


@pytest.mark.parametrize("cache", [pk.PK_F8, pk.PK_BF16])
@pytest.mark.parametrize("n, top, most, Hq, Hkv, d, page", [
    (300, 200, 3, 16, 8, 64, 16),        # a wave for a request, 16 rows and fewer
    (97, 180, 7, 32, 8, 128, 16),        # 28 rows
    (70, 150, 9, 64, 8, 128, 32),        # 72 rows: three waves for a request
    (90, 2500, 1, 32, 8, 128, 16),       # pieces of several kinds, merged in the launch
    (90, 2500, 7, 32, 8, 64, 16),        # 28 rows, merged behind it
    (80, 1500, 11, 64, 8, 128, 48),      # 88 rows
    (40, 4000, 2, 16, 8, 128, 16),       # more than half of a round
    (620, 300, 2, 8, 1, 64, 16),         # more requests than are read at once
    (3, 20000, 4, 4, 1, 128, 64),        # hundreds of pieces of one request
    (5, 3000, 64, 16, 1, 64, 16),        # 1024 rows
    (33, 900, 17, 8, 8, 128, 16),        # 17 rows
])
def test_batches_of_every_kind(n, top, most, Hq, Hkv, d, page, cache):
    ctx, drafts = ragged(n + most, n, top, most)
    s = step.make(n, ctx, drafts, Hq, Hkv, d, page, cache)
    mask = step.masks(s, "tree")
    ws = pk.new_tree_workspace(n, most, Hq, Hkv, d)
    first = step.call(s, mask, ws=ws)
    chain = step.call(s, None, torch.float32, ws=ws)
    again = step.call(s, mask, ws=ws)
    torch.cuda.synchronize()
    assert torch.equal(first, again)                               # joined in one order, whoever comes last
    dense(s, mask, first)
    dense(s, None, chain)


@pytest.mark.parametrize("cache", [pk.PK_F8, pk.PK_BF16])
@pytest.mark.parametrize("n, top, most, Hq, Hkv, d", [(100, 60, 20, 40, 8, 64), (80, 100, 17, 64, 8, 128), (70, 4, 64, 16, 8, 64), (90, 0, 33, 32, 8, 128)])
def test_many_short_trees(n, top, most, Hq, Hkv, d, cache):
    """Tables of 256 keys and fewer: no request has two pieces.  Two chunks of rows, a second one of a few rows, contexts of nothing."""
    ctx, drafts = ragged(3 * n, n, top, most)
    s = step.make(most, ctx, drafts, Hq, Hkv, d, 16, cache)
    assert s["table"].shape[1] * 16 <= 256
    for kind in ("tree", "bits"):
        mask = step.masks(s, kind)
        dense(s, mask, step.call(s, mask))


@pytest.mark.parametrize("Hq, Hkv, drafts", [(8, 8, 2), (16, 4, 6), (32, 2, 12)])
def test_the_width_of_the_table_changes_no_result_beyond_rounding(Hq, Hkv, drafts):
    """A wide table allows long requests, so that a launch is laid out for them; the requests are the same short ones."""
    s = step.make(7, [30 + 2 * i for i in range(80)], [drafts] * 80, Hq, Hkv, 64, 16, pk.PK_F8)
    mask = step.masks(s, "bits")
    dense(s, mask, step.call(s, mask))
    s["table"] = torch.cat([s["table"], torch.full((80, 500), 1 << 30, dtype=torch.int32, device=DEV)], 1).contiguous()
    dense(s, mask, step.call(s, mask))


@pytest.mark.parametrize("Hq, drafts", [(8, 4), (16, 8), (40, 10)])
def test_a_captured_call_with_merges_replays(Hq, drafts):
    n = 12
    s = step.make(61, [4000 - 300 * i for i in range(n)], [drafts] * n, Hq, 2, 128, 16, pk.PK_F8)
    full = list(s["lens"])
    dev = lambda x: torch.from_numpy(np.ascontiguousarray(x)).to(DEV)  # noqa: E731
    q_start, lens, out = dev(s["q_start"]), dev(np.array(full, np.int32)), torch.zeros_like(s["q"])
    ws = pk.new_tree_workspace(n, drafts, Hq, 2, 128)
    args = (s["c"], s["q"], q_start, drafts, None, s["table"], lens, out, s["scale"], ws)
    pk.tree_attn(*args)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        pk.tree_attn(*args)
    for now in (full, [max(drafts, x // 7) for x in full], [drafts] * n, full):
        lens.copy_(torch.tensor(now, dtype=torch.int32))
        out.fill_(7.0)
        graph.replay()
        torch.cuda.synchronize()
        eager = torch.full_like(out, 5.0)
        pk.tree_attn(*args[:7], eager, *args[8:])
        torch.cuda.synchronize()
        assert torch.equal(out, eager)
    dense(s, None, out)


@pytest.mark.parametrize("cache", [pk.PK_F8, pk.PK_BF16])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("Hkv, d, page", [(8, 128, 16), (3, 64, 48)])
@pytest.mark.parametrize("fused", [False, True])
def test_runs_of_slots_at_every_offset(Hkv, d, page, cache, dtype, fused):
    """Runs of 1..13 tokens from every place of a cell on, backwards ones, and slots that no pool has between them."""
    g, rng = step.gen(d), np.random.default_rng(Hkv)
    runs, at = [], 0
    for length in list(range(1, 14)) * 4:
        at += int(rng.integers(0, 6))
        r = np.arange(at, at + length)
        runs.append(r[::-1] if rng.random() < 0.15 else r)
        at += length
        if rng.random() < 0.3:
            runs.append(np.array([-1 if rng.random() < 0.5 else 1 << 40]))
    order = rng.permutation(len(runs))
    slots = np.concatenate([runs[i] for i in order]).astype(np.int64)
    blocks = at // page + 1
    t = step.TYPES[dtype]
    c = pk.new_kv_cache(blocks, page, Hkv, d, cache)
    for x in (c.k, c.v) + ((c.scales,) if cache == pk.PK_F8 else ()):
        x.view(torch.uint8).fill_(0x31)
    k, v = (step.randn(g, len(slots), Hkv, d, dtype=t) for _ in "kv")
    old = step.token_major(c)
    where = torch.from_numpy(slots).to(DEV)
    if fused:
        q = step.randn(g, len(slots), 2 * Hkv, d, dtype=t)
        qo = torch.empty_like(q)
        pk.qkv_cache_write(c, q, k, v, where, qo, None, None, 1e-6, None)
        assert torch.equal(q, qo)
    else:
        pk.kv_cache_write(c, k, v, where)
    got, ok = step.token_major(c), (slots >= 0) & (slots < blocks * page)
    for i, x in enumerate((k, v)):
        want, scale = old[i].copy(), old[2 + i].copy()
        if cache == pk.PK_F8:
            codes, E = oc.quantize(step.f64(x))
            want[slots[ok]], scale[slots[ok]] = codes[ok], 2.0 ** E[ok]
        else:
            want[slots[ok]] = step.f64(x.to(torch.bfloat16))[ok]
        assert np.array_equal(got[i], want) and np.array_equal(got[2 + i], scale)


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("Hkv, d, rot", [(8, 128, 128), (4, 64, 32)])
@pytest.mark.parametrize("cache", [pk.PK_F8, pk.PK_BF16])
def test_normed_keys_have_the_codes_of_the_exact_value(Hkv, d, rot, cache, interleaved):
    """Arithmetic in 64 bits and one rounding: nothing falls on the other side of a middle."""
    g, tokens, page = step.gen(rot), 700, 16
    c = pk.new_kv_cache(tokens // page + 1, page, Hkv, d, cache)
    q, k, v = (step.randn(g, tokens, Hkv, d) for _ in "qkv")
    w = step.randn(g, d)
    table, pos = step.table_of(4096, rot), torch.randint(0, 4096, (tokens,), generator=g, device=DEV, dtype=torch.int32)
    pk.qkv_cache_write(c, q, k, v, torch.arange(tokens, device=DEV), torch.empty_like(q), w, w, 2.0 ** -20, pk.Rope(table, pos, None, interleaved))
    want = oc.norm_rope(step.f64(k), step.f64(w), 2.0 ** -20, step.f64(table), pos.cpu().numpy()[None], None, interleaved)
    kc, _, ks, _ = step.token_major(c)
    if cache == pk.PK_F8:
        codes, E = oc.quantize(want)
        assert np.array_equal(kc[:tokens], codes) and np.array_equal(ks[:tokens], 2.0 ** E)
    else:
        # nearest in 8 bits of fraction, ties to even: numpy has no such type, so the distance says it
        assert (np.abs(kc[:tokens] - want) <= 2.0 ** (np.floor(np.log2(np.abs(want))) - 8) * (1 + 1e-12)).all()


@pytest.mark.parametrize("cache", [pk.PK_F8, pk.PK_BF16])
@pytest.mark.parametrize("T, kept, page", [(64, 64, 16), (64, 33, 48), (40, 17, 16), (9, 8, 32), (1, 1, 16)])
def test_many_kept_tokens(T, kept, page, cache):
    n = 5
    s = step.make(T, [0, 3, 16, 77, 200], [T] * n, 8, 3 if T < 10 else 2, 64, page, cache, hostile=False) if T < 10 else \
        step.make(T, [0, 3, 16, 77, 200], [T] * n, 8, 2, 128, page, cache, hostile=False)
    rng = np.random.default_rng(kept)
    keep = np.stack([np.sort(rng.permutation(T)[:kept]) for _ in range(n)]).astype(np.int32)
    count = np.array([kept, kept, 0, 1, kept + 100], np.int32)
    keep[1, -1] = 1 << 20                                          # no drafted token: passed over
    before = step.token_major(s["c"])
    dev = lambda x: torch.from_numpy(np.ascontiguousarray(x)).to(DEV)  # noqa: E731
    new = torch.zeros(n, dtype=torch.int32, device=DEV)
    pk.kv_cache_keep(s["c"], s["table"], dev(np.array(s["lens"], np.int32)), dev(s["q_start"]), dev(keep), dev(count), new)
    torch.cuda.synchronize()
    now = min(kept, T)
    want = [x.copy() for x in before]
    for i in range(n):
        base = s["lens"][i] - T
        for j in range(min(int(count[i]), now)):
            f = int(keep[i, j])
            if f < T:
                for x, y in zip(want, before):
                    x[s["slots"][i][base + j]] = y[s["slots"][i][base + f]]
    for x, y in zip(step.token_major(s["c"]), want):
        assert np.array_equal(x, y, equal_nan=True)
    assert new.tolist() == [s["lens"][i] - T + min(int(count[i]), now, T) for i in range(n)]


@pytest.mark.parametrize("cache, blocks", [(pk.PK_F8, 290_000), (pk.PK_BF16, 150_000)])
def test_a_cache_of_more_than_four_gib(cache, blocks):
    """Every call on the last pages of a cache whose K and V are longer than 2^32 bytes each, against the same pages of a small one."""
    g, Hkv, d, page, n, T = step.gen(9), 8, 128, 16, 3, 5
    far, near = pk.new_kv_cache(blocks, page, Hkv, d, cache), pk.new_kv_cache(12, page, Hkv, d, cache)
    assert far.k.nbytes > 1 << 32
    table = torch.arange(12, dtype=torch.int32, device=DEV).view(n, 4).flip(0).contiguous()
    lens = torch.tensor([64, 37, 20], dtype=torch.int32, device=DEV)
    rows = step.randn(g, 12 * page, Hkv, d), step.randn(g, 12 * page, Hkv, d)
    q, w = step.randn(g, n * T, 16, d), step.randn(g, d)
    q_start = torch.arange(0, n * T + 1, T, dtype=torch.int32, device=DEV)
    rope = pk.Rope(step.table_of(64, d), torch.arange(n * T, dtype=torch.int32, device=DEV))
    keep = torch.tensor([[1, 3], [0, 4], [2, 3]], dtype=torch.int32, device=DEV)
    results = []
    for c, first in ((near, 0), (far, blocks - 12)):
        slots = torch.arange(12 * page, device=DEV) + first * page
        pk.kv_cache_write(c, *rows, slots)
        at = table + first
        new = torch.cat([at[i].long()[(torch.arange(T, device=DEV) + int(lens[i]) - T) // page] * page + (torch.arange(T, device=DEV) + int(lens[i]) - T) % page for i in range(n)])
        qo, out, after = torch.empty_like(q), torch.empty_like(q), torch.empty_like(lens)
        pk.qkv_cache_write(c, q, rows[0][:n * T], rows[1][:n * T], new, qo, w, w, 1e-6, rope)
        pk.tree_attn(c, qo, q_start, T, None, at, lens, out, d ** -0.5, pk.new_tree_workspace(n, T, 16, Hkv, d))
        pk.kv_cache_keep(c, at, lens, q_start, keep, torch.full_like(lens, 2), after)
        k, v = (torch.zeros(128, Hkv, d, device=DEV) for _ in "kv")
        pk.kv_cache_read(c, at, after, torch.tensor([0, 64, 101], dtype=torch.int32, device=DEV), k, v)
        results.append((qo, out, after, k, v))
    for x, y in zip(*results):
        assert torch.equal(x, y)
    assert (results[0][3] != 0).any() and (results[0][1] != 0).any()
