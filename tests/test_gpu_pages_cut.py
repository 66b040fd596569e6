"""Requests that are cut to fewer tokens behind a fork, as a search that goes back does: pk_kv_pages_select gives up the pages behind their tokens, and nothing that another
request holds is written afterwards."""
import numpy as np
import pytest

from paper_2602_06072_amd import binding as pk
from tests.test_gpu_pages import Batch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n, cut", [(2, [16, 9]), (6, None), (1100, None)])
def test_no_shared_page_is_written_by_requests_that_were_cut(n, cut):
    page, rng = 16, np.random.default_rng(n)
    b = Batch(rng, max(1, n // 4), 12, 8 * n + 60, page, 130)
    b.lens[:] = np.maximum(b.lens, 1)
    b.pages[:] = np.maximum(b.pages, 1)
    b.refs[:] = 0
    blocks, at = rng.permutation(len(b.refs)), 0
    for i in range(len(b.lens)):
        b.table[i, :b.pages[i]] = blocks[at:at + b.pages[i]]
        b.refs[b.table[i, :b.pages[i]]] = 1
        at += b.pages[i]
    ws = pk.new_pages_workspace(len(b.refs))
    b.select(np.sort(rng.integers(0, len(b.lens), n)).astype(np.int32))           # forks
    whole = b.lens.copy()
    b.lens[::2] = np.minimum(cut if cut else rng.integers(0, whole.max() + 1, n), whole)[::2]
    b.select(np.arange(n, dtype=np.int32))                         # what was cut gives up its pages
    assert np.array_equal(b.pages, -(-b.lens // page))
    grow = rng.integers(1, 40, n).astype(np.int32)
    served, src, dst = b.reserve(grow, ws)
    assert served.all()
    for i in range(n):
        first, last = b.lens[i] // page, min(-(-(b.lens[i] + grow[i]) // page), b.most)
        assert (b.refs[b.table[i, first:last]] == 1).all()
    assert ((src >= 0) == (dst >= 0)).all()
