"""Attention over pages that requests share, against the definition in 64 bits and against pk_tree_attn.

Tolerances are those of the attention of drafted tokens (tests/test_gpu_cache_step.py): probabilities are rounded to bf16, 2^-8 of
sum p |v| above and below the fraction, and a bf16 output by 2^-8 of itself.  Joining the shared part with a request's own part adds some
roundings of 2^-24.  Two calls that sum in another order differ by twice that at most."""
import numpy as np
import pytest
import torch

from paper_2602_06072_amd import binding as pk
from tests.test_gpu_cache_step import check, gen, masks, placement, randn, random_cache

pytestmark = pytest.mark.gpu
DEV = "cuda"


def dev(x):
    return torch.from_numpy(np.ascontiguousarray(x)).to(DEV)


def make(seed, families, Hq, Hkv, d, page, cache, front=(), back=(), hostile=True, roomy=True):
    """families: [(prefix, [(own tokens, drafted tokens), ...]), ...]; front, back: requests that are in none.  The whole pages of a prefix are
    shared; places where no token of a request is hold NaN.  roomy: a block table with room for 300 MB of keys and values, as shared pages are
    looked for from 256 MB on; below, every request is taken alone."""
    g, rng = gen(seed), np.random.default_rng(seed)
    requests = [(0, o, t) for o, t in front] + [(p, o, t) for p, m in families for o, t in m] + [(0, o, t) for o, t in back]
    start = np.concatenate([[0], np.cumsum([len(m) for _, m in families])]).astype(np.int32) + len(front)
    lens, drafts = [p + o + t for p, o, t in requests], [t for _, _, t in requests]
    blocks = sum((x + page - 1) // page for x in lens) + 3
    c = random_cache(g, blocks, page, Hkv, d, cache, 0.3)
    table, slots = placement(rng, lens, page, blocks)
    host = table.cpu().numpy()
    at = len(front)
    for p, m in families:
        for i in range(at + 1, at + len(m)):
            host[i, :p // page] = host[at, :p // page]
        at += len(m)
    if roomy:
        columns = int(300e6 / (len(lens) * page * 2 * Hkv * (d + 1 if cache == pk.PK_F8 else 2 * d))) + 1
        host = np.concatenate([host, rng.integers(-(1 << 30), 1 << 30, (len(lens), max(0, columns - host.shape[1])), dtype=np.int32)], 1)
    slots = [host[i, np.arange(x) // page].astype(np.int64) * page + np.arange(x) % page for i, x in enumerate(lens)]
    if hostile:
        used = np.zeros(blocks * page, bool)
        for x in slots:
            used[x] = True
        free = dev(np.nonzero(~used)[0])
        nan = torch.full((len(free), Hkv, d), float("nan"), device=DEV)
        pk.kv_cache_write(c, nan, nan, free)
        if cache == pk.PK_F8:
            c.scales.view(torch.uint8)[free // page, :, :, free % page] = 255
    q_start = np.concatenate([[0], np.cumsum(drafts)]).astype(np.int32)
    return dict(c=c, table=dev(host), slots=slots, lens=lens, drafts=drafts, q_start=q_start, q=randn(g, int(q_start[-1]), Hq, d), max_q=max(drafts + [0]),
                scale=d ** -0.5, rng=rng, family_start=start)


def call(s, mask, out_dtype=torch.bfloat16, ws=None, stream=None, family_start=None, max_q=None):
    out = torch.full(s["q"].shape, 7.0, dtype=out_dtype, device=DEV)
    c, max_q = s["c"], s["max_q"] if max_q is None else max_q
    if ws is None:
        ws = pk.new_shared_tree_workspace(len(s["lens"]), max_q, s["q"].shape[0], s["q"].shape[1], c.Hkv, c.d)
    pk.shared_tree_attn(c, s["q"], dev(s["q_start"]), max_q, None if mask is None else dev(mask.view(np.int64)), s["table"],
                        dev(np.array(s["lens"], np.int32)), dev(s["family_start"] if family_start is None else np.array(family_start, np.int32)), out, s["scale"],
                        ws, stream=stream)
    torch.cuda.synchronize()
    return out


HEADS = [(8, 2, 64), (8, 8, 128), (7, 1, 128), (32, 4, 128), (32, 1, 64)]
BATCHES = [
    dict(families=[(100, [(3, 1), (0, 1)])]),
    dict(families=[(0, [(5, 2), (70, 1)]), (63, [(1, 1)] * 3), (64, [(0, 1)] * 3)]),
    dict(families=[(700, [(3, 1), (64, 2), (300, 1), (0, 5)]), (333, [(9, 1)])], front=[(20, 1), (200, 3)], back=[(130, 2)]),
    dict(families=[(1500, [(i, 1) for i in range(40)])]),
    dict(families=[(257, [(5, 64), (80, 33)]), (640, [(0, 17), (17, 1), (1, 0)])]),
    dict(families=[(400, [(0, 1)] * 5), (400, [(100, 0)] * 3), (100, [(0, 3), (0, 0)])]),
    dict(families=[(3000, [(4, 1), (9, 1)])]),
    dict(families=[(130 + 20 * i, [(i, 1 + i % 3)] * (1 + i % 4)) for i in range(30)]),
]


@pytest.mark.parametrize("Hq, Hkv, d", HEADS)
@pytest.mark.parametrize("batch", range(len(BATCHES)))
@pytest.mark.parametrize("kind, cache, page", [("tree", pk.PK_F8, 16), ("chain", pk.PK_F8, 48), ("bits", pk.PK_BF16, 32)])
def test_shared_attention(Hq, Hkv, d, batch, kind, cache, page):
    b = BATCHES[batch]
    s = make(batch + Hq, b["families"], Hq, Hkv, d, page, cache, b.get("front", ()), b.get("back", ()))
    if sum(s["drafts"]) * Hq * max(s["lens"]) > 4e6:
        s = make(batch + Hq, b["families"], Hq // Hkv, 1, d, page, cache, b.get("front", ()), b.get("back", ()))           # (the oracle's time)
    mask = masks(s, kind)
    check(s, mask, call(s, mask, torch.float32 if kind == "bits" else torch.bfloat16))


def test_tables_of_little_room():
    for batch in BATCHES[:3]:
        s = make(11, batch["families"], 8, 2, 128, 16, pk.PK_F8, batch.get("front", ()), batch.get("back", ()), roomy=False)
        mask = masks(s, "tree")
        got = call(s, mask, torch.float32)
        check(s, mask, got)
        assert torch.equal(got, as_alone(s, mask))


def as_alone(s, mask, out_dtype=torch.float32):
    c = s["c"]
    out = torch.full(s["q"].shape, 7.0, dtype=out_dtype, device=DEV)
    pk.tree_attn(c, s["q"], dev(s["q_start"]), s["max_q"], None if mask is None else dev(mask.view(np.int64)), s["table"], dev(np.array(s["lens"], np.int32)), out,
                 s["scale"], pk.new_tree_workspace(len(s["lens"]), s["max_q"], s["q"].shape[1], c.Hkv, c.d))
    return out


def near(a, b):
    """Two fp32 results that differ in the order of sums: each is off by 2^-8 (sum p |v| + |o|), |v| is at most 6 or so here."""
    assert torch.isfinite(a).all() == torch.isfinite(b).all()
    err = (a - b).abs().max().item()
    assert err <= 2 * 2.0 ** -8 * 8, err
    assert (a - b).norm().item() <= 4e-3 * b.norm().item()          # (errors of 2^-9 in the mean that are independent: 2e-3 each)


@pytest.mark.parametrize("Hq, Hkv, d, cache", [(32, 8, 128, pk.PK_F8), (64, 8, 128, pk.PK_F8), (64, 8, 64, pk.PK_BF16), (16, 16, 128, pk.PK_F8), (40, 8, 64, pk.PK_F8), (28, 4, 128, pk.PK_BF16)])
@pytest.mark.parametrize("shape", ["many", "long", "trees", "mixed"])
def test_large_batches_equal_the_attention_of_each(Hq, Hkv, d, cache, shape):
    rng = np.random.default_rng(Hq)
    families = {"many": [(2100, [(int(rng.integers(0, 400)), 1) for _ in range(130)])],
                "long": [(30011, [(int(rng.integers(0, 900)), 1 + i % 2) for i in range(5)]), (9000, [(7, 1)] * 2)],
                "trees": [(int(rng.integers(100, 3000)), [(int(rng.integers(0, 300)), int(rng.integers(1, 33))) for _ in range(6)]) for _ in range(9)],
                "mixed": [(int(rng.integers(0, 4000)), [(int(rng.integers(0, 2000)), int(rng.integers(0, 5))) for _ in range(int(rng.integers(1, 9)))]) for _ in range(60)]}[shape]
    s = make(Hq + d, families, Hq, Hkv, d, 16, cache, hostile=False)
    mask = masks(s, "tree")
    near(call(s, mask, torch.float32), as_alone(s, mask))


def test_whatever_the_families_are():
    """Requests that share nothing, a part of what others share, or less than their drafted tokens leave over, and families that overlap nothing or
    everything: the result is that of each request alone."""
    s = make(1, [(640, [(70, 2), (0, 3), (200, 1), (5, 1)]), (320, [(64, 2), (900, 1)])], 16, 4, 128, 16, pk.PK_F8, front=[(300, 1)], back=[(40, 1), (650, 2)])
    mask = masks(s, "tree")
    n = len(s["lens"])
    for family_start in ([0, n], [0], [n], [1, 7], [0, 2, 4, 6, n], [3, 3, 3, n], list(range(n + 1)), [0, 0, n, n], [-5, 3, 100], [7, 2, 5], [1 << 30, -(1 << 30)]):
        check(s, mask, call(s, mask, torch.float32, family_start=family_start))
    # a member that ends inside the shared pages, its drafted tokens among them, and one without any token
    t = make(2, [(1000, [(10, 2), (300, 1), (0, 2), (40, 1)])], 16, 4, 128, 16, pk.PK_F8)
    for i, x in ((1, 500), (3, 0)):
        t["lens"][i] = x
        t["slots"][i] = t["slots"][i][:x]
    check(t, masks(t, "chain"), call(t, None, torch.float32))
    t["lens"][2] = 1                                               # fewer tokens than drafted ones
    got = call(t, None, torch.float32)
    near(got, as_alone(t, None))


def test_pages_that_differ_and_come_together_again():
    s = make(3, [(2000, [(100, 1), (100, 2), (100, 1)])], 8, 2, 64, 16, pk.PK_F8)
    host = s["table"].cpu().numpy()
    host[1, 70], host[2, 5] = host[1, 130], host[0, 3]             # (the second one's 71st page is another one, the third one's 6th)
    s["table"] = dev(host)
    s["slots"] = [host[i, np.arange(x) // 16].astype(np.int64) * 16 + np.arange(x) % 16 for i, x in enumerate(s["lens"])]
    mask = masks(s, "tree")
    check(s, mask, call(s, mask, torch.float32))


def test_numbers_that_are_not_finite_in_shared_and_in_hidden_places():
    s = make(4, [(500, [(30, 3), (90, 2)])], 8, 2, 128, 16, pk.PK_BF16)
    c = s["c"]
    k = torch.randn(3, 2, 128, device=DEV)
    v = torch.randn(3, 2, 128, device=DEV)
    v[0, 0, 5], v[1, 1, 7], v[2, 0, 9] = float("inf"), float("nan"), float("-inf")
    pk.kv_cache_write(c, k, v, dev(np.array([s["slots"][0][10], s["slots"][0][200], s["slots"][1][-1]], np.int64)))
    mask = masks(s, "chain")
    check(s, mask, call(s, mask, torch.float32))                   # (close() asks for the same NaNs and infinities)


def test_tables_without_numbers_behind_the_pages_and_lengths_beyond_the_table():
    s = make(5, [(320, [(20, 1), (50, 1)] * 210)], 8, 8, 128, 16, pk.PK_F8, hostile=False, roomy=False)
    cut = s["table"][:, :22].contiguous()                          # 352 tokens
    lens = [min(x, 352) for x in s["lens"]]
    s["table"] = cut
    got = call(dict(s, lens=[x + 1000 * (x > 352) for x in s["lens"]]), None, torch.float32)
    want = as_alone(dict(s, lens=[x + 1000 * (x > 352) for x in s["lens"]]), None)
    near(got, want)
    assert lens[0] == 341


def test_results_repeat_and_one_workspace_serves_all_calls():
    ws = pk.new_shared_tree_workspace(200, 40, 3000, 64, 8, 128)
    rng = np.random.default_rng(6)
    for seed in range(6):
        families = [(int(rng.integers(0, 3000)), [(int(rng.integers(0, 500)), int(rng.integers(0, 9 if seed % 2 else 2))) for _ in range(int(rng.integers(1, 12)))])
                    for _ in range(int(rng.integers(1, 12)))]
        s = make(seed, families, 64 if seed % 3 else 32, 8, 128 if seed % 2 else 64, 16, pk.PK_F8, hostile=False)
        if s["max_q"] == 0:
            continue
        mask = masks(s, "tree")
        first = call(s, mask, torch.float32, ws=ws)
        assert torch.equal(first, call(s, mask, torch.float32, ws=ws))
        assert torch.equal(first, call(s, mask, torch.float32))
        near(first, as_alone(s, mask))


def test_rows_behind_the_last_request_and_without_a_request_stay():
    s = make(7, [(200, [(9, 2), (30, 1)])], 8, 2, 64, 16, pk.PK_F8)
    q = torch.cat([s["q"], s["q"]])
    s["q"] = q
    out = call(s, None)
    assert (out[3:] == 7).all() and not (out[:3] == 7).all()
    out = call(s, None, max_q=1)
    assert (out[1] == 7).all() and not (out[0] == 7).all()


def test_replays_of_a_captured_call_and_another_stream():
    s = make(8, [(900, [(i * 20, 1 + i % 4) for i in range(9)]), (64, [(1, 1)] * 4)], 32, 8, 128, 16, pk.PK_F8, hostile=False)
    mask = masks(s, "tree")
    want = call(s, mask)
    stream = torch.cuda.Stream()
    assert torch.equal(call(s, mask, stream=stream), want)
    c, n = s["c"], len(s["lens"])
    lens, q, out, table = dev(np.array(s["lens"], np.int32)), s["q"].clone(), torch.zeros_like(s["q"]), s["table"].clone()
    q_start, family, words = dev(s["q_start"]), dev(s["family_start"]), dev(mask.view(np.int64))
    ws = pk.new_shared_tree_workspace(n, 4, q.shape[0], 32, 8, 128)
    run = lambda: pk.shared_tree_attn(c, q, q_start, 4, words, table, lens, family, out, s["scale"], ws)  # noqa: E731
    run()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run()
    for turn in range(4):
        out.zero_()
        less = turn * 37
        new = [max(4, x - less) for x in s["lens"]]
        lens.copy_(dev(np.array(new, np.int32)))
        q.copy_(s["q"] * (1 + turn))
        family.copy_(dev(s["family_start"] if turn % 2 == 0 else np.array([0, 3, n], np.int32)))
        graph.replay()
        torch.cuda.synchronize()
        t = dict(s, lens=new, q=s["q"] * (1 + turn))
        assert torch.equal(out, call(t, mask, family_start=family.cpu().numpy()))
        near(out.float(), as_alone(t, mask))


def test_places_behind_four_gib():
    """A pool of bf16 keys of more than 4 GiB, shared pages at its end."""
    blocks, page, Hkv, d = 34000, 64, 8, 128
    c = pk.new_kv_cache(blocks, page, Hkv, d, pk.PK_BF16)
    rng = np.random.default_rng(9)
    lens, prefix = [700, 645, 900], 640
    table = np.zeros((3, 500), np.int32)
    table[:, :10] = blocks - 10 + np.arange(10)
    table[:, 10:15] = blocks - 40 + np.arange(15).reshape(3, 5)
    table[:, 15:] = blocks - 1
    g = gen(9)
    used = torch.from_numpy(np.unique(table)).long().to(DEV)
    slots = (used[:, None] * page + torch.arange(page, device=DEV)).reshape(-1)
    pk.kv_cache_write(c, torch.randn(len(slots), Hkv, d, generator=g, device=DEV), torch.randn(len(slots), Hkv, d, generator=g, device=DEV), slots)
    s = dict(c=c, table=dev(table), lens=lens, drafts=[1, 1, 1], q_start=np.arange(4).astype(np.int32), q=randn(g, 3, 32, d), max_q=1, scale=d ** -0.5,
             family_start=np.array([0, 3], np.int32), rng=rng)
    got = call(s, None, torch.float32)
    near(got, as_alone(s, None))
    small = pk.new_kv_cache(40, page, Hkv, d, pk.PK_BF16)
    for x, y in ((small.k, c.k), (small.v, c.v)):
        x.copy_(y[blocks - 40:])
    t = dict(s, c=small, table=dev(np.where(table >= blocks - 40, table - (blocks - 40), 0).astype(np.int32)))
    assert torch.equal(got, call(t, None, torch.float32)) and prefix == 640
