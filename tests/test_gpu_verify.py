"""Judging of drafted tokens on the device against oracle/branch.py.  Answers are whole numbers and have to be equal: both sides
compute in 64 bits, a draw falls between two borders that their roundings move by 1e-15 or so, and there are some 1e5 borders and 1e4 draws
here, so that a test that fails for it has a chance of 1e-6."""
import numpy as np
import pytest
import torch

from oracle import branch as ob
from paper_2602_06072_amd import binding as pk

pytestmark = pytest.mark.gpu
DEV = "cuda"
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def dev(x, t=None):
    return torch.from_numpy(np.ascontiguousarray(x)).to(DEV, t)


def make(seed, sizes, vocab, dtype, drawn, tree, spread=2.0, pad=0, hot=None):
    """A batch on the host and on the device.  Drafted tokens are drawn from the draft, or are likely ones."""
    rng = np.random.default_rng(seed)
    total = int(sum(sizes))
    width = vocab + pad
    base = rng.normal(size=(total, width)) * spread
    t = TYPES[dtype]
    target = torch.from_numpy(base).to(t)
    draft = torch.from_numpy(base + 0.7 * rng.normal(size=base.shape)).to(t)
    q_start = np.concatenate([[0], np.cumsum(sizes)]).astype(np.int32)
    temperature = rng.uniform(0.5, 1.5, len(sizes)).astype(np.float32) if hot is None else np.full(len(sizes), hot, np.float32)
    tokens, words = np.zeros(total, np.int32), np.zeros(total, np.uint64)
    for i, T in enumerate(sizes):
        own = []
        for s in range(T):
            p = s - 1 if not tree or s == 0 else int(rng.integers(max(0, s - 6), s))
            own.append((1 << s) | (own[p] if s else 0))
            row = (draft if drawn else target)[q_start[i] + max(p, 0), :vocab].double().numpy()
            w = ob.probabilities(row, max(float(temperature[i]), 0.2))
            tokens[q_start[i] + s] = rng.choice(vocab, p=w / w.sum()) if vocab > 1 else 0
        words[q_start[i]:q_start[i + 1]] = own
    return dict(target=target, draft=draft if drawn else None, vocab=vocab, tokens=tokens, q_start=q_start, sizes=list(sizes), mask=words if tree else None,
                temperature=temperature, accept=rng.random(total).astype(np.float32), sample=rng.random(len(sizes)).astype(np.float32), max_q=max(list(sizes) + [0]))


def call(s, max_keep=None, ws=None, stream=None, max_q=None):
    n, total = len(s["sizes"]), len(s["tokens"])
    k = s["max_q"] if max_keep is None else max_keep
    keep, count, after = (torch.full(x, -9, dtype=torch.int32, device=DEV) for x in ((n, max(1, k)), (n,), (n,)))
    ws = pk.new_verify_workspace(n, total, s["vocab"]) if ws is None else ws
    cut = lambda x: None if x is None else x.to(DEV)[:, :s["vocab"]]  # noqa: E731
    pk.draft_verify(cut(s["target"]), cut(s["draft"]), dev(s["tokens"]), dev(s["q_start"]), s["max_q"] if max_q is None else max_q,
                    None if s["mask"] is None else dev(s["mask"].view(np.int64)), None if s["temperature"] is None else dev(s["temperature"]),
                    dev(s["accept"]), dev(s["sample"]), keep, count, after, ws, stream=stream)
    torch.cuda.synchronize()
    return keep.cpu().numpy(), count.cpu().numpy(), after.cpu().numpy()


def check(s, got, max_keep=None, max_q=64):
    keep, count, after = got
    k = max(1, s["max_q"] if max_keep is None else max_keep)
    for i, T in enumerate(s["sizes"]):
        a, b = s["q_start"][i], s["q_start"][i] + min(T, max_q)
        cut = lambda x: None if x is None else x[a:b, :s["vocab"]].double().numpy()  # noqa: E731
        kept, next_token = ob.draft_verify(cut(s["target"]), cut(s["draft"]), s["tokens"][a:b], None if s["mask"] is None else s["mask"][a:b],
                                           1.0 if s["temperature"] is None else float(s["temperature"][i]), s["accept"][a:b], s["sample"][i], k)
        assert count[i] == len(kept) and keep[i].tolist() == kept + [-1] * (k - len(kept)) and after[i] == next_token, (i, T, kept, next_token, keep[i], after[i])


@pytest.mark.parametrize("vocab", [1, 2, 7, 8, 2047, 2048, 2049, 5003, 40001])
@pytest.mark.parametrize("dtype, drawn, tree", [("bf16", True, True), ("f32", True, False), ("bf16", False, True), ("f32", False, True)])
def test_judging(vocab, dtype, drawn, tree):
    s = make(vocab, [1, 5, 0, 64, 17, 2, 33, 1], vocab, dtype, drawn, tree)
    check(s, call(s))
    check(s, call(s, 2), 2)


@pytest.mark.parametrize("dtype, spread", [("bf16", 2.0), ("f32", 2.0), ("bf16", 0.0), ("f32", 40.0)])
def test_chains_of_many_logits(dtype, spread):
    s = make(1, [64, 5, 1, 40, 64, 2, 0, 30], 50001, dtype, True, False, spread=spread)            # 206 rows: more than 2^23 logits, whose first sums have 32 bits
    s["target"][3, ::7], s["draft"][5, 1::9] = float("nan"), -float("inf")
    check(s, call(s))
    s["temperature"][:4] = 0.0, 0.01, 5.0, 1e-20
    check(s, call(s))
    check(s, call(s, 3), 3)


@pytest.mark.parametrize("dtype, sizes, vocab", [("bf16", [64], 130001), ("f32", [12, 3, 0, 20, 1], 70001), ("bf16", [2, 1, 9], 16385), ("bf16", [40] * 6, 66003), ("f32", [7], 8193)])
def test_few_trees_with_long_rows(dtype, sizes, vocab):
    """Tokens with siblings whose rows several workgroups share."""
    s = make(vocab, sizes, vocab, dtype, True, True, spread=0.7)
    for turn in range(3):
        got = call(s)
        check(s, got)
        s["temperature"][turn % len(sizes)] = (0.0, 0.3, 1e-25)[turn]
        s["accept"][1::2] = 0.9999                                 # (most are refused)


@pytest.mark.parametrize("case", ["chain", "many", "lookup", "tree"])
def test_choices_next_to_a_border(case):
    """u is the fp32 number next to the border, off it by 3e-8 or less (and by 1e-11 hardly ever): 64 bits decide."""
    drawn, tree, vocab = case in ("chain", "many"), case == "tree", 45007 if case == "many" else 3001
    s = make(2, [2] * (100 if case == "many" else 60), vocab, "f32", drawn, tree)
    for i in range(len(s["sizes"])):
        a = s["q_start"][i]
        x, t = s["tokens"][a + 1], float(s["temperature"][i])
        border = ob.probabilities(s["target"][a].double().numpy(), t)[x]
        if drawn:
            border /= ob.probabilities(s["draft"][a].double().numpy(), t)[x]
        s["accept"][a + 1] = np.float32(border)
    got = call(s)
    check(s, got)
    assert 0.2 < (got[1] == 2).mean() < 0.95


@pytest.mark.parametrize("sizes", [[1], [0], [], [2], [64] * 3, [1] * 300, [3, 0, 9] * 30])
@pytest.mark.parametrize("drawn", [True, False])
def test_batches(sizes, drawn):
    s = make(len(sizes), sizes, 301, "bf16", drawn, True)
    check(s, call(s))


@pytest.mark.parametrize("spread", [0.0, 0.01, 30.0, 1000.0])
def test_flat_and_steep_rows(spread):
    for dtype in TYPES:
        s = make(3, [1, 9, 30], 9001, dtype, True, True, spread=spread)
        check(s, call(s))


@pytest.mark.parametrize("hot", [0.0, -1.0, float("nan"), 1e-30, 1e-3, 100.0, float("inf")])
def test_temperatures(hot):
    s = make(5, [1, 6, 20], 3001, "bf16", True, True, hot=hot if hot == hot else 0.0)
    s["temperature"][:] = hot
    if not hot > 0:                                                # drafted tokens that are the largest logits, of which there are several
        s["target"][:, 100:2900:7] = s["target"].max() + 1
        s["tokens"][::2] = 100
    check(s, call(s))
    s["temperature"] = None
    check(s, call(s))


def test_rows_apart_and_rows_of_every_alignment():
    for pad in (0, 1, 5, 40):
        s = make(pad, [4, 1, 11, 8], 1013, "bf16", True, False, pad=pad)
        s["target"][:, 1013:], s["draft"][:, 1013:] = float("inf"), float("nan")       # between the rows
        check(s, call(s))


def test_numbers_that_are_not_finite():
    s = make(6, [6] * 40, 700, "f32", True, True)
    rng = np.random.default_rng(6)
    for x in (s["target"], s["draft"]):
        x[torch.from_numpy(rng.random(x.shape) < 0.5)] = -float("inf")
        x[torch.from_numpy(rng.random(x.shape) < 0.05)] = float("nan")
        x[5:30:3, 17:19] = float("inf")
    s["target"][60:72], s["draft"][66:80] = -float("inf"), float("nan")
    s["target"][90, :] = float("nan")
    s["tokens"][100:140:3] = 17
    check(s, call(s))
    s["draft"] = None
    check(s, call(s))
    s["temperature"][:] = 0
    check(s, call(s))


def test_random_numbers_at_the_ends():
    for u, v in ((0.0, 0.0), (1 - 2.0 ** -24, 1 - 2.0 ** -24), (1.0, 1.0), (2.0, -1.0)):
        for drawn in (True, False):
            s = make(7, [1, 8, 21], 4099, "bf16", drawn, True)
            s["target"][:, :50] = -float("inf")
            s["accept"][:], s["sample"][:] = u, v
            check(s, call(s))
    s["accept"][:] = float("nan")                                  # nothing stays
    keep, count, _ = call(s)
    assert (count == 1).all()


def test_tokens_outside_of_the_vocabulary_and_the_same_token_twice():
    for drawn in (True, False):
        s = make(8, [9, 9, 9], 500, "f32", drawn, False)
        s["mask"] = np.array([1] + [1 | 1 << t for t in range(1, 9)] * 1, np.uint64).repeat(1)
        s["mask"] = np.concatenate([s["mask"]] * 3)                # all drafted ones are children of the first
        s["tokens"][1:9] = [-1, 500, 3, 3, 3, 1 << 30, 4, 3]
        s["tokens"][10:18] = int(s["target"][9].argmax())
        s["accept"][:18] = 0.999
        check(s, call(s))


def test_masks_without_parents_and_bits_from_outside():
    s = make(9, [12] * 6, 90, "f32", True, True)
    rng = np.random.default_rng(9)
    s["mask"] = rng.integers(0, 1 << 63, 72, dtype=np.uint64) * 2 + 1                  # parents anywhere, bits of tokens that there are not
    s["mask"][:12] = 0
    s["mask"][12:24] &= ~np.uint64(1)                              # no way to the first token
    s["accept"] *= 0.2
    check(s, call(s))


@pytest.mark.parametrize("max_keep", [1, 2, 5, 100])
def test_no_more_than_max_keep(max_keep):
    s = make(10, [1, 20, 64], 400, "bf16", True, False)
    s["draft"] = s["target"].clone()                               # all would stay
    got = call(s, max_keep)
    check(s, got, max_keep)
    assert got[1].tolist() == [1, min(20, max_keep), min(64, max_keep)]


def test_max_q_below_a_requests_tokens():
    s = make(11, [1, 20, 9], 400, "bf16", True, True)
    check(s, call(s, max_q=5), max_q=5)
    keep, count, after = call(s, max_q=0)
    assert (keep == -1).all() and (count == 0).all() and (after == -1).all()


def test_one_workspace_for_all_calls_and_results_that_repeat():
    ws = pk.new_verify_workspace(300, 2000, 50000)
    for seed, sizes, vocab in ((1, [8] * 200, 2500), (2, [1], 50000), (3, [64] * 10, 4000), (4, [3, 5], 17)):
        for drawn in (True, False):
            s = make(seed, sizes, vocab, "bf16", drawn, True)
            first = call(s, ws=ws)
            check(s, first)
            for a, b in zip(first, call(s, ws=ws)):
                assert np.array_equal(a, b)


def test_rows_behind_four_gib():
    total, vocab = 20000, 120001                                   # 4.8 GB of logits
    target = torch.zeros(total, vocab, dtype=torch.bfloat16, device=DEV)
    target[-3:] = -30.0
    target[-1, 77], target[-2, 120000], target[-3, 5] = 9.0, 9.0, 9.0
    q_start = dev(np.array([0, 0, total - 3, total], np.int32))
    tokens = torch.zeros(total, dtype=torch.int32, device=DEV)
    tokens[-2:] = torch.tensor([5, 120000], dtype=torch.int32, device=DEV)
    u = torch.full((total,), 0.5, device=DEV)
    keep, count, after = (torch.full(x, -9, dtype=torch.int32, device=DEV) for x in ((3, 4), (3,), (3,)))
    pk.draft_verify(target, None, tokens, q_start, 3, None, None, u, u[:3], keep, count, after, pk.new_verify_workspace(3, total, vocab))
    torch.cuda.synchronize()
    # Request 1 has its first three tokens looked at: rows of equal logits.  Its token 1, number 0 of the vocabulary, is refused (1 / 120001 < 0.5) and has no weight
    # any more: number k has k behind it of 120000 equal weights, and k > 0.5 * 120000 first holds for 60001.
    assert count.tolist() == [0, 1, 3] and keep[2].tolist() == [0, 1, 2, -1] and after.tolist() == [-1, 60001, 77]


def test_replays_of_a_captured_call_and_another_stream():
    s = make(12, [5, 1, 30, 12], 3000, "bf16", True, True)
    other = make(13, [5, 1, 30, 12], 3000, "bf16", True, True)
    stream = torch.cuda.Stream()
    check(s, call(s, stream=stream))
    n, total = 4, len(s["tokens"])
    ws = pk.new_verify_workspace(n, total, 3000)
    buf = {k: (x.to(DEV) if isinstance(x, torch.Tensor) else dev(x.view(np.int64) if k == "mask" else x)) for k, x in s.items()
           if k in ("target", "draft", "tokens", "mask", "temperature", "accept", "sample")}
    q_start = dev(s["q_start"])
    keep, count, after = (torch.full(x, -9, dtype=torch.int32, device=DEV) for x in ((n, 30), (n,), (n,)))
    run = lambda: pk.draft_verify(buf["target"], buf["draft"], buf["tokens"], q_start, 30, buf["mask"], buf["temperature"], buf["accept"], buf["sample"],  # noqa: E731
                                  keep, count, after, ws)
    run()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run()
    for x in (other, s, other):
        for k, y in buf.items():
            y.copy_(x[k] if isinstance(x[k], torch.Tensor) else torch.from_numpy(x[k].view(np.int64) if k == "mask" else x[k]))
        graph.replay()
        torch.cuda.synchronize()
        check(x, (keep.cpu().numpy(), count.cpu().numpy(), after.cpu().numpy()))
        assert call(x)[2].tolist() == after.tolist()               # (eager work in between)


def test_the_next_tokens_are_distributed_as_the_target():
    """8000 requests with one row of logits: tokens behind token 0, whether they come from a child or from what is left, against the target's
    probabilities.  A share of 8000 draws is off by 5 standard deviations at most (chance 6e-7 each, 24 tokens)."""
    n, vocab, rng = 8000, 24, np.random.default_rng(14)
    p, q = rng.normal(size=vocab) * 1.5, rng.normal(size=vocab) * 1.5
    P, Q = ob.probabilities(p, 1.0), ob.probabilities(q, 1.0)
    for kids, drawn in ((1, True), (3, True), (2, False)):
        T = kids + 1
        tokens = np.zeros((n, T), np.int32)
        tokens[:, 1:] = rng.choice(vocab, size=(n, kids), p=Q) if drawn else [3, 11][:kids]
        s = dict(target=torch.from_numpy(np.tile(p, (n * T, 1))).float(), draft=torch.from_numpy(np.tile(q, (n * T, 1))).float() if drawn else None, vocab=vocab,
                 tokens=tokens.reshape(-1), q_start=np.arange(0, n * T + 1, T).astype(np.int32), sizes=[T] * n,
                 mask=np.tile(np.array([1] + [1 | 2 << t for t in range(kids)], np.uint64), n), temperature=np.ones(n, np.float32),
                 accept=rng.random(n * T).astype(np.float32), sample=rng.random(n).astype(np.float32), max_q=T)
        keep, count, after = call(s)
        got = np.where(count > 1, tokens[np.arange(n), np.maximum(keep[:, 1], 0)], after)
        share = np.bincount(got, minlength=vocab) / n
        assert (np.abs(share - P) < 5 * np.sqrt(P * (1 - P) / n) + 1e-6).all()
