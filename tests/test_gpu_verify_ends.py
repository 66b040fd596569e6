"""Judging of drafted tokens where nothing is left of a row, and in a workspace of a larger batch.  Whole numbers, which have to equal oracle/branch.py's."""
import numpy as np
import pytest
import torch

from paper_2602_06072_amd import binding as pk
from tests.test_gpu_verify import call, check, make

pytestmark = pytest.mark.gpu


def with_few_tokens(seed, sizes, vocab, dtype, drawn, finite):
    """Every row has logits of 0 at the places `finite`, of which every drafted token is one (in turns), and none elsewhere."""
    s = make(seed, sizes, vocab, dtype, drawn, True)
    s["target"][:] = -float("inf")
    s["target"][:, finite] = 0.0
    if drawn:
        s["draft"] = s["target"].clone()
    words = [1 | 2 << t for t in range(max(sizes) - 1)]            # all of them are children of the first
    s["mask"] = np.concatenate([np.array(([1] + words)[:T], np.uint64) for T in sizes])
    for a, T in zip(s["q_start"], sizes):
        s["tokens"][a + 1:a + T] = [finite[t % len(finite)] for t in range(T - 1)]
    return s


@pytest.mark.parametrize("u", [1.0, float("nan")])
@pytest.mark.parametrize("finite", [[17], [3, 250]])
@pytest.mark.parametrize("vocab", [301, 50001])
@pytest.mark.parametrize("dtype, drawn", [("bf16", False), ("f32", False), ("f32", True)])
def test_refused_tokens_that_held_all_of_the_row(u, finite, vocab, dtype, drawn):
    """1 > 1 * 1 and 1/2 > 1 * 1/2 are false, as anything over a NaN is: both are refused, nothing is left, and the token behind is drawn from the whole row.
    (Logits of 0 have weights of 1 on both sides, so that these probabilities are exact.)"""
    s = with_few_tokens(vocab, [3, 2, 5, 3, 1], vocab, dtype, drawn, finite)
    s["accept"][:] = u
    s["sample"][:] = [0.1, 0.9, 0.6, 0.4, 0.5]
    got = call(s)
    check(s, got)
    assert set(got[2].tolist()) <= set(finite)
    if len(finite) == 1 or u != u:
        assert (got[1] == 1).all()


def quick(seed, sizes, vocab):
    """A chain for each request, whose drafted tokens are the likeliest of the target's row in front of them, or any."""
    rng = np.random.default_rng(seed)
    total = sum(sizes)
    target = torch.from_numpy(rng.normal(size=(total, vocab)).astype(np.float32) * 4).bfloat16()
    tokens = rng.integers(0, vocab, total).astype(np.int32)
    tokens[1:] = np.where(rng.random(total - 1) < 0.8, target.float().argmax(1)[:-1].numpy(), tokens[1:])
    return dict(target=target, draft=None, vocab=vocab, tokens=tokens, q_start=np.concatenate([[0], np.cumsum(sizes)]).astype(np.int32), sizes=sizes, mask=None,
                temperature=np.full(len(sizes), 0.4, np.float32), accept=rng.random(total).astype(np.float32), sample=rng.random(len(sizes)).astype(np.float32),
                max_q=max(sizes))


def test_a_row_of_which_no_number_is_left_and_none_was():
    s = with_few_tokens(1, [3, 1], 400, "bf16", False, [9])
    s["target"][:] = -float("inf")
    s["accept"][:] = 1.0
    got = call(s)
    check(s, got)
    assert (got[2] == -1).all()


@pytest.mark.parametrize("vocab, sizes, smaller", [(128256, [1] * 35 + [32], [[1] * 34 + [32], [2] * 3]), (32000, [8] * 257, [[8] * 256, [64] * 12]),
                                                   (128256, [9] * 11 + [1], [[8] * 8, [1]]), (262145, [2, 3], [[1], [2, 2]])])
def test_a_workspace_of_the_largest_batch_serves_smaller_ones(vocab, sizes, smaller):
    ws = pk.new_verify_workspace(len(sizes), sum(sizes), vocab)
    for x in [sizes] + smaller:
        s = quick(vocab, x, vocab)
        check(s, call(s, ws=ws))
    assert not ws[:65536 * 4].any()                                # counts of arrivals: ready for the next call


def test_outputs_between_the_rows():
    """Rows apart from one another leave room that is nobody's: outputs may be there."""
    s = quick(3, [3, 1, 4, 2], 500)
    room = torch.full((10, 540), float("nan"), device="cuda")
    room[:, :500] = s["target"].float()
    words = room.view(torch.int32)
    flat = lambda row, n: words[row, 500:500 + n]  # noqa: E731
    keep, count, after = flat(2, 16).view(4, 4), flat(0, 4), flat(9, 4)
    dev = lambda x: torch.from_numpy(x).cuda()  # noqa: E731
    pk.draft_verify(room[:, :500], None, dev(s["tokens"]), dev(s["q_start"]), 4, None, dev(s["temperature"]), dev(s["accept"]), dev(s["sample"]), keep, count, after,
                    pk.new_verify_workspace(4, 10, 500))
    torch.cuda.synchronize()
    check(s, (keep.cpu().numpy(), count.cpu().numpy(), after.cpu().numpy()))
    with pytest.raises(pk.PackInferError, match="keep_count overlaps target"):
        pk.draft_verify(room[:, :500], None, dev(s["tokens"]), dev(s["q_start"]), 4, None, dev(s["temperature"]), dev(s["accept"]), dev(s["sample"]), keep,
                        words[4, 497:501], after, pk.new_verify_workspace(4, 10, 500))
    assert torch.equal(room[:, :500].cpu(), s["target"].float())
