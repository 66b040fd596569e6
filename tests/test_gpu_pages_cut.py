"""Requests that are cut to fewer tokens behind a fork, as a search that goes back does: nothing that another request holds is written when they grow again."""
import numpy as np
import pytest

from paper_2602_06072_amd import binding as pk
from tests.test_gpu_pages import Batch

pytestmark = pytest.mark.gpu


def forked(n, spare, seed, page=16, extra=0):
    """n requests, forks of n // 4 others, in a pool with room for `spare` more blocks."""
    rng = np.random.default_rng(seed)
    m = max(1, n // 4)
    b = Batch(rng, m, 12, m * 12 + spare, page, 130)
    b.lens[:] = np.maximum(b.lens, 1)
    b.pages[:] = np.minimum(-(-b.lens // page) + rng.integers(0, extra + 1, m), b.most)
    b.refs[:] = 0
    blocks, at = rng.permutation(len(b.refs)), 0
    for i in range(m):
        b.table[i, :b.pages[i]] = blocks[at:at + b.pages[i]]
        b.refs[b.table[i, :b.pages[i]]] = 1
        at += b.pages[i]
    b.select(np.sort(rng.integers(0, m, n)).astype(np.int32))
    return b, rng


def cut(b, rng, to=None):
    """Every second request to the length `to`, or to any."""
    whole = b.lens.copy()
    b.lens[::2] = np.minimum(to if to else rng.integers(0, whole.max() + 1, len(whole)), whole)[::2]


def held(b):
    count = np.zeros(len(b.refs), np.int64)
    for i in range(len(b.lens)):
        np.add.at(count, b.table[i, :b.pages[i]], 1)
    return count


def grow(b, rng, ws, most=40):
    """Reserves; says what was served.  What a served request is to write is its own then, and what anyone's tokens are in stays where it is, or is copied."""
    n, page = len(b.lens), b.page
    before, more = b.table.copy(), rng.integers(0, most, n).astype(np.int32)
    served, src, dst = b.reserve(more, ws)
    assert np.array_equal(held(b), b.refs)
    for i in range(n):
        first, whole, last = b.lens[i] // page, -(-b.lens[i] // page), min(-(-(b.lens[i] + more[i]) // page), b.most)
        same = b.table[i, :whole] == before[i, :whole]
        assert same[:first].all() and (same.all() or (src[i] == before[i, first] and dst[i] == b.table[i, first]))
        if served[i] and more[i] > 0:
            assert (b.refs[b.table[i, first:last]] == 1).all()
            b.lens[i] = min(b.lens[i] + more[i], last * page)
    return served


@pytest.mark.parametrize("n, to", [(2, 16), (2, 9), (2, 32), (6, None), (40, None), (1100, None)])
@pytest.mark.parametrize("trimmed", [False, True])
def test_no_shared_page_is_written_by_requests_that_were_cut(n, to, trimmed):
    """trimmed: pk_kv_pages_select gives up what is behind their tokens; without, pk_kv_pages_reserve does where it matters."""
    b, rng = forked(n, 6 * n + 20, n)
    ws = pk.new_pages_workspace(len(b.refs))
    for turn in range(3):
        cut(b, rng, to)
        if trimmed:
            b.select(np.arange(n, dtype=np.int32))
            assert np.array_equal(b.pages, -(-b.lens // b.page))
        grow(b, rng, ws)
        b.select(rng.integers(0, n, n).astype(np.int32))


def test_the_page_at_a_border_and_pages_further_behind():
    """Two requests on five pages; one is cut to two whole pages, or into its third."""
    for length, more, keeps, copied in ((32, 1, 2, False), (32, 100, 2, False), (37, 5, 5, True), (37, 20, 3, True), (80, 3, 5, False), (0, 1, 0, False), (32, 0, 5, False)):
        b = Batch(np.random.default_rng(1), 1, 8, 30, 16, 16)
        b.lens[:], b.pages[:], b.table[0, :5] = 80, 5, [9, 4, 22, 7, 13]
        b.refs[:] = 0
        b.refs[[9, 4, 22, 7, 13]] = 1
        b.select(np.array([0, 0], np.int32))
        b.lens[1] = length
        served, src, dst = b.reserve(np.array([0, more], np.int32), pk.new_pages_workspace(30))
        assert served.all() and (src[1] == 22) == copied and src[0] == -1
        assert b.table[0, :5].tolist() == [9, 4, 22, 7, 13]
        want = [9, 4, 22, 7, 13][:keeps]
        want[2:3] = [dst[1]] if copied else want[2:3]
        assert b.table[1, :keeps].tolist() == want
        assert b.pages[1] == max(keeps, min(8, -(-(length + more) // 16)) if more else 0)
        assert np.array_equal(held(b), b.refs)


@pytest.mark.parametrize("n, spare", [(24, 10), (1300, 400)])
def test_blocks_that_run_out_for_requests_that_were_cut(n, spare):
    b, rng = forked(n, spare, n)
    ws = pk.new_pages_workspace(len(b.refs))
    b.refs[b.refs == 0] = np.where(np.arange((b.refs == 0).sum()) < spare, 0, 1 << 20)            # (a caller holds the others)
    kept_by_caller = b.refs >= 1 << 20
    cut(b, rng)
    before = b.table.copy(), b.lens.copy(), b.pages.copy()
    more = rng.integers(0, 40, n).astype(np.int32)
    served, _, _ = b.reserve(more, ws)
    assert 0 < served.sum() < n
    for i in np.nonzero(served == 0)[0]:
        assert np.array_equal(b.table[i], before[0][i]) and b.pages[i] == before[2][i]
    assert np.array_equal(held(b)[~kept_by_caller], b.refs[~kept_by_caller])


def test_room_that_was_reserved_stays():
    """Pages behind the tokens that nobody else holds are used, not handed back."""
    b, rng = forked(1, 60, 5, extra=3)
    ws = pk.new_pages_workspace(len(b.refs))
    b.reserve(np.array([60], np.int32), ws)
    pages, table = b.pages.copy(), b.table.copy()
    b.reserve(np.array([33], np.int32), ws)
    assert np.array_equal(b.pages, pages) and np.array_equal(b.table, table)
