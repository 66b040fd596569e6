"""Lengths and numbers on the device that no program means: the calls stay inside of their tables and leave the cache as it is."""
import numpy as np
import pytest
import torch

from paper_2602_06072_amd import binding as pk
from tests import test_gpu_cache_step as step

pytestmark = pytest.mark.gpu
LEAST, MOST = -(1 << 31), (1 << 31) - 1


@pytest.mark.parametrize("cache", [pk.PK_F8, pk.PK_BF16])
@pytest.mark.parametrize("kv_len, q_start", [(LEAST, [0, 9]), (LEAST + 3, [0, 9]), (MOST, [0, 9]), (MOST, [9, 0]), (-1, [0, 9]), (4, [0, 9]), (40, [0, MOST]), (40, [LEAST, MOST]), (40, [MOST, LEAST])])
def test_keep_with_lengths_out_of_range_moves_nothing(kv_len, q_start, cache):
    """In 64 bits no kept token of these has a place in front of the first token or a source inside of the table."""
    s = step.make(3, [40, 40], [9, 9], 4, 2, 64, 16, cache, hostile=False)
    dev = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    keep, count = dev([[1, 3, 5, 7, 8], [0, 1, 2, 3, 4]]), dev([5, 0])
    before, new = step.token_major(s["c"]), dev([7, 7])
    pk.kv_cache_keep(s["c"], s["table"], dev([kv_len, 49]), dev(q_start + [q_start[1]]), keep, count, new)
    torch.cuda.synchronize()
    base = kv_len - (q_start[1] - q_start[0])
    kept = min(5, max(0, q_start[1] - q_start[0]))
    moves = [j for j in range(kept) if base + j >= 0 and base + int(keep[0, j]) < s["table"].shape[1] * 16]
    assert not moves
    for a, b in zip(before, step.token_major(s["c"])):
        assert np.array_equal(a, b, equal_nan=True)
    assert new.tolist() == [(base + kept + (1 << 31)) % (1 << 32) - (1 << 31), 49]
