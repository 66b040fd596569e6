"""The calls of branching and judging together, as examples/branching_decode.py makes them: forked answers that share their prompt's pages, drafted
tokens judged on the device, steps replayed from a graph."""
import numpy as np
import pytest
import torch

from examples import branching_decode as bd
from paper_2602_06072_amd import binding as pk

pytestmark = pytest.mark.gpu
HEADS = (8, 2, 64)


def cached(model, batch, sequences):
    """Keys and values of the batch's tokens as they are cached, and those of the same sequences written as prompts of a new batch."""
    rows = sum(map(len, sequences))
    start = torch.tensor(np.concatenate([[0], np.cumsum([len(x) for x in sequences])[:-1]]), dtype=torch.int32, device="cuda")
    fresh = bd.Batch(model, sum(len(x) // bd.PAGE + 1 for x in sequences) + 1, max(len(x) // bd.PAGE + 1 for x in sequences), batch.n, dtype=batch.cache.dtype)
    bd.prompts(model, fresh, sequences)
    out = []
    for b in (batch, fresh):
        k, v = (torch.full((rows, model.Hkv, model.d), 7.0, device="cuda") for _ in "kv")
        pk.kv_cache_read(b.cache, b.table, b.lens, start, k, v)
        out.append((k, v))
    torch.cuda.synchronize()
    return out


@pytest.mark.parametrize("roomy", [1, 60])
@pytest.mark.parametrize("dtype", [pk.PK_F8, pk.PK_BF16])
def test_what_stays_is_what_was_drawn(dtype, roomy):
    """roomy: the table has room for so much that shared pages are looked for."""
    model, batch, sequences, new, _ = bd.generate(5, 6, 12, 3, HEADS, prompt=(20, 700), seed=3, dtype=dtype, roomy=roomy)
    assert batch.lens.tolist() == [len(x) for x in sequences]
    assert any(len(x) > 14 for x in new) and len({tuple(x) for x in new}) > 20         # drafted tokens stay, and answers differ
    used = int((batch.refs > 0).sum())
    assert used == sum(-(-len(x) // bd.PAGE) for x in sequences) and bool((batch.refs[:used] == 1).all())
    for a, b in zip(*cached(model, batch, sequences)):
        assert torch.equal(a, b)


def test_replayed_steps_equal_eager_ones():
    runs = [bd.generate(3, 5, 8, 2, HEADS, prompt=(30, 300), seed=4, graph=graph, roomy=100) for graph in (True, False)]
    assert runs[0][3] == runs[1][3]
    for a, b in zip(runs[0][2], runs[1][2]):
        assert np.array_equal(a, b)
    assert torch.equal(runs[0][1].table, runs[1][1].table) and torch.equal(runs[0][1].refs, runs[1][1].refs)


def test_a_pool_that_is_too_small_is_noticed():
    with pytest.raises(AssertionError, match="too small"):
        bd.generate(2, 6, 30, 3, HEADS, prompt=(20, 100), seed=5, spare=0.4)


def test_two_batches_on_two_streams():
    """Steps of two batches, each with caches and workspaces of its own, enqueued in turns on two streams: the same answers as alone."""
    alone = [bd.generate(2, 4, 5, 2, HEADS, prompt=(40, 200), seed=s, graph=False, roomy=150)[3] for s in (6, 7)]
    streams, made = [torch.cuda.Stream() for _ in range(2)], []
    for s, stream in zip((6, 7), streams):
        with torch.cuda.stream(stream):
            made.append(bd.generate(2, 4, 5, 2, HEADS, prompt=(40, 200), seed=s, graph=False, roomy=150)[3])
    assert made == alone
