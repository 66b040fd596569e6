"""The example of prompts and speculative decoding: what it accepted must be what the same tokens give as one prompt."""
import importlib.util
import os

import numpy as np
import pytest
import torch

from paper_2602_06072_amd import binding as pk

pytestmark = pytest.mark.gpu
PATH = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "speculative_decode.py")


def example():
    spec = importlib.util.spec_from_file_location("speculative_decode", PATH)
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


@pytest.mark.parametrize("n, steps, drafts, heads, dtype", [(5, 6, 9, (8, 2, 128), pk.PK_F8), (3, 4, 1, (4, 4, 64), pk.PK_BF16), (2, 5, 40, (8, 1, 64), pk.PK_F8)])
def test_accepted_tokens_equal_one_long_prompt(n, steps, drafts, heads, dtype):
    """Every request's prompt and accepted tokens as one prompt of a new layer: the cache has the same codes, and the outputs are the
    same within the rounding of probabilities and outputs to bf16 (2^-8 of the sum of p |v| each, from either side)."""
    m = example()
    layer, lens, rows, first, accepted, context, _ = m.generate(n, steps, drafts, heads, 3, (1, 70), dtype)
    assert [int(x) for x in context] == [int(x) + sum(len(a[0]) for a in acc) for x, acc in zip(lens, accepted)]
    ends = np.cumsum(lens)
    whole = torch.cat([torch.cat([rows[e - x:e]] + [a[0] for a in acc]) for e, x, acc in zip(ends, lens, accepted)])
    want_out = torch.cat([torch.cat([first[e - x:e]] + [a[1] for a in acc]) for e, x, acc in zip(ends, lens, accepted)])
    again = m.Layer(n, int(layer.block_table.shape[1]) * m.PAGE, heads, 3, dtype)
    got = m.prefill(again, whole, context)
    start = torch.from_numpy(np.concatenate([[0], np.cumsum(context)[:-1]]).astype(np.int32)).cuda()
    read = []
    for y in (layer, again):
        k, v = (torch.empty(int(context.sum()), y.Hkv, y.d, device="cuda") for _ in "kv")
        pk.kv_cache_read(y.cache, y.block_table, torch.from_numpy(context.astype(np.int32)).cuda(), start, k, v)
        read.append((k, v))
    assert torch.equal(read[0][0], read[1][0]) and torch.equal(read[0][1], read[1][1])
    top = read[0][1].abs().amax()                                  # no sum of p |v| is larger
    assert float((got.float() - want_out.float()).abs().max()) <= 6 * 2.0 ** -8 * float(top)
    # and on the whole: errors of single rows are of either sign
    assert float((got.float() - want_out.float()).norm() / want_out.float().norm()) < 2.0 ** -7
