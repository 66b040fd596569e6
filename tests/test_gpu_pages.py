"""Pages of a batch on the device (forking, reserving, compacting) and copies of blocks, against oracle/branch.py: whole numbers
and bytes, which have to be equal."""
import numpy as np
import pytest
import torch

from oracle import branch as ob
from paper_2602_06072_amd import binding as pk

pytestmark = pytest.mark.gpu
DEV = "cuda"


def dev(x):
    return torch.from_numpy(np.ascontiguousarray(x, np.int32)).to(DEV)


def host(*x):
    torch.cuda.synchronize()
    return [y.cpu().numpy() for y in x]


class Batch:
    """A batch on the host, its rows full of numbers that are no blocks behind their pages."""

    def __init__(self, rng, n, most, blocks, page, longest, extra=0):
        self.page, self.most = page, most
        self.table = rng.integers(-(1 << 30), 1 << 30, (n, most)).astype(np.int32)
        self.lens = rng.integers(0, longest + 1, n).astype(np.int32)
        self.pages = np.minimum(-(-self.lens // page) + (rng.integers(0, extra + 1, n) if extra else 0), most).astype(np.int32)
        self.refs, perm, at = np.zeros(blocks, np.int32), rng.permutation(blocks), 0
        for i in range(n):
            self.pages[i] = min(self.pages[i], blocks - at)
            self.lens[i] = min(self.lens[i], self.pages[i] * page)
            self.table[i, :self.pages[i]] = perm[at:at + self.pages[i]]
            at += self.pages[i]
        self.refs[perm[:at]] = 1

    def select(self, rows_from, ws=None):
        """The new batch, by both; equal in everything."""
        m = len(rows_from)
        new = np.full((m, self.most), 7, np.int32)
        t, ls, ps, refs = dev(new), dev(np.full(m, -9)), dev(np.full(m, -9)), dev(self.refs)
        old = dev(self.table), dev(self.lens), dev(self.pages)
        pk.kv_pages_select(*old, dev(rows_from), t, ls, ps, refs, self.page)
        lens, pages = ob.pages_select(self.table, self.lens, self.pages, rows_from, new, self.refs, self.page)
        got = host(t, ls, ps, refs, *old)
        for g, want in zip(got, (new, lens, pages, self.refs, self.table, self.lens, self.pages)):
            assert np.array_equal(g, want)
        self.table, self.lens, self.pages = new, lens, pages

    def reserve(self, grow, ws):
        n = len(self.lens)
        t, ps, refs = dev(self.table), dev(self.pages), dev(self.refs)
        served, src, dst = (dev(np.full(n, -9)) for _ in range(3))
        pk.kv_pages_reserve(t, dev(self.lens), ps, dev(grow), refs, self.page, served, src, dst, ws)
        want = ob.pages_reserve(self.table, self.lens, self.pages, grow, self.refs, self.page)
        for g, w in zip(host(t, ps, refs, served, src, dst), (self.table, self.pages, self.refs) + want):
            assert np.array_equal(g, w)
        assert not ws.view(torch.int32).view(-1, 3136)[:, :2048].any()                 # ready for the next call, of whatever size
        return want

    def compact(self, moves, ws, in_place=False):
        t, refs = dev(self.table), dev(self.refs)
        nt, nr = t if in_place else t.clone(), torch.empty_like(refs)
        src, dst = dev(np.full(moves, -9)), dev(np.full(moves, -9))
        pk.kv_pages_compact(t, dev(self.pages), refs, nt, nr, src, dst, ws)
        want = ob.pages_compact(self.table, self.pages, self.refs, moves)
        for g, w in zip(host(nt, nr, src, dst), want):
            assert np.array_equal(g, w)
        self.table, self.refs = want[0], want[1]
        return want[2:]


@pytest.mark.parametrize("n, most, blocks, page, longest, extra", [(1, 1, 1, 16, 16, 0), (3, 9, 40, 16, 120, 2), (70, 30, 3000, 16, 460, 5),
                                                                  (257, 7, 900, 48, 330, 3), (1500, 3, 5000, 64, 190, 1), (2, 400, 9000, 16, 6000, 9)])
@pytest.mark.parametrize("tight", [False, True])
def test_steps_of_forking_and_growing(n, most, blocks, page, longest, extra, tight):
    """Steps as a search makes them: requests fork, some end, all grow; with few blocks some are not served."""
    rng = np.random.default_rng(n + most)
    b = Batch(rng, n, most, blocks if not tight else max(1, int(n * longest / page * 0.55)), page, longest, extra)
    ws = pk.new_pages_workspace(len(b.refs))
    for step in range(4):
        m = max(1, int(n * rng.uniform(0.5, 1.6)))
        b.select(rng.integers(-1, len(b.lens) + 1, m))
        grow = rng.integers(-1, rng.choice([2, 5, 3 * page]), m).astype(np.int32)
        served, src, _ = b.reserve(grow, ws)
        b.lens = np.where((served == 1) & (grow > 0), np.minimum(b.lens + np.maximum(grow, 0), b.pages * page), b.lens).astype(np.int32)
        held = np.zeros(len(b.refs), np.int64)
        for i in range(m):
            np.add.at(held, b.table[i, :b.pages[i]], 1)
        assert np.array_equal(held, b.refs)                        # nothing is lost, nothing is held twice
    b.compact(int((b.refs > 0).sum()) + 3, ws, in_place=bool(n % 2))
    used = int((b.refs > 0).sum())
    assert (b.refs[:used] > 0).all() and not b.refs[used:].any()


def test_rows_of_many_entries():
    rng = np.random.default_rng(6)
    b = Batch(rng, 3, 33001, 70000, 16, 16 * 33001)
    b.lens[:], b.pages[:] = np.minimum(b.lens, [16 * 33001, 16 * 20000 - 5, 16 * 255]), np.minimum(b.pages, [33001, 20000, 255])
    b.refs[:] = 0
    for i in range(3):
        np.add.at(b.refs, b.table[i, :b.pages[i]], 1)
    ws = pk.new_pages_workspace(70000)
    b.select([1, 0, 1, 2])
    b.reserve(np.array([40, 0, 700, 3], np.int32), ws)
    b.select([3, 0, 2])
    b.compact(50000, ws, in_place=True)


def test_a_page_stays_with_the_last_of_its_holders():
    page, ws = 16, pk.new_pages_workspace(64)
    for n, writers in ((5, [0, 1, 2, 3, 4]), (5, [1, 2]), (5, [4]), (2000, list(range(2000)))):
        blocks = n + 3
        rng = np.random.default_rng(n)
        b = Batch(rng, 1, 2, blocks, page, 16)
        b.lens[:], b.pages[:], b.table[0, 0] = 5, 1, 1
        b.refs[:] = 0
        b.refs[1] = 1
        b.select([0] * n)
        grow = np.zeros(n, np.int32)
        grow[writers] = 1
        served, src, dst = b.reserve(grow, pk.new_pages_workspace(blocks) if blocks > 64 else ws[:pk.lib().pk_kv_pages_workspace_bytes(blocks)])
        assert served.all() and (src >= 0).sum() == (n - 1 if len(writers) == n else len(writers))


def test_pages_run_out_in_the_order_of_requests():
    page = 16
    b = Batch(np.random.default_rng(3), 3, 4, 12, page, 16)
    b.lens[:], b.pages[:] = [16, 5, 16], 1
    b.table[:, 0] = [3, 8, 1]
    b.refs[:] = 0
    b.refs[[3, 8, 1]] = 1
    b.select([0, 1, 1, 2, 0])
    # 9 blocks are free: 3, then 1 for a copy and 3, then 2 of the 3 that the next one wants; what needs none is served, a keeper is not
    served, src, _ = b.reserve(np.array([48, 60, 3, 48, 0], np.int32), pk.new_pages_workspace(12))
    assert served.tolist() == [1, 1, 1, 0, 1] and src.tolist() == [-1, 8, -1, -1, -1]
    b = Batch(np.random.default_rng(3), 1, 4, 3, page, 16)
    b.lens[:], b.pages[:], b.table[0, 0] = 5, 1, 2
    b.refs[:] = [1, 1, 1]
    b.select([0, 0])
    served, src, _ = b.reserve(np.array([1, 1], np.int32), pk.new_pages_workspace(3))
    assert served.tolist() == [0, 0] and src.tolist() == [-1, -1]  # the second one must not write what the first still reads


@pytest.mark.parametrize("large, small", [(700, 300), (5000, 1300), (5000, 40)])
def test_one_workspace_for_pools_of_several_sizes(large, small):
    rng, ws = np.random.default_rng(large), pk.new_pages_workspace(large)
    for turn in range(3):
        for blocks in (small, large, large):
            n = blocks // 20
            b = Batch(rng, n, 8, blocks, 16, 90)
            b.select(np.repeat(np.arange(n), 2)[rng.permutation(2 * n)])
            b.reserve(rng.integers(0, 30, 2 * n).astype(np.int32), ws)
            b.compact(blocks, ws)
            b.reserve(rng.integers(0, 30, 2 * n).astype(np.int32), ws)


def test_blocks_that_a_caller_holds_and_numbers_outside_of_the_pool():
    page, ws = 16, pk.new_pages_workspace(9)
    b = Batch(np.random.default_rng(4), 2, 5, 9, page, 70)
    b.table[:], b.lens[:], b.pages[:] = [[6, -3, 99, 1, 0], [5, 6, 7, 7, 7]], [50, 20], [4, 2]
    b.refs[:] = [0, 1, 3, 0, 0, 1, 2, 0, 0]                        # (block 2: held from outside)
    b.select([1, 0, 1])
    b.reserve(np.array([3, 20, 0], np.int32), ws)
    b.compact(9, ws)


@pytest.mark.parametrize("blocks, part, moves", [(1, 0.0, 1), (1, 1.0, 0), (5, 0.4, 9), (4096, 0.5, 4096), (4097, 0.99, 300), (30011, 0.3, 30011), (12288, 0.0, 5),
                                                 (12288, 1.0, 5), (70001, 0.5, 1000)])
def test_compaction(blocks, part, moves):
    rng = np.random.default_rng(blocks)
    n, most = 20, max(1, blocks // 10)
    b = Batch(rng, n, most, blocks, 16, int(32 * part * blocks / n))
    while True:
        left = int((b.refs[int((b.refs > 0).sum()):] > 0).sum())
        src, dst = b.compact(moves, pk.new_pages_workspace(blocks))
        assert (src >= 0).sum() == min(left, moves) and not set(src[src >= 0]) & set(dst[dst >= 0])
        if left <= moves or moves == 0:
            break


@pytest.mark.parametrize("cache", [pk.PK_F8, pk.PK_BF16])
@pytest.mark.parametrize("Hkv, d, page, count", [(8, 128, 16, 3), (1, 64, 16, 700), (5, 128, 48, 40), (2, 64, 128, 1), (8, 128, 16, 600)])
def test_copies_of_blocks(Hkv, d, page, count, cache):
    g, rng = torch.Generator(device=DEV).manual_seed(count), np.random.default_rng(count)
    blocks = 2 * count + 5

    def filled(k):
        c = pk.new_kv_cache(k, page, Hkv, d, cache)
        for x in (c.k, c.v, c.scales):
            if x is not None:
                y = x.view(torch.uint8).view(-1)
                y.copy_(torch.randint(0, 256, y.shape, generator=g, device=DEV, dtype=torch.uint8))
        return c

    c, other = filled(blocks), filled(count + 9)
    perm = rng.permutation(blocks)
    src, dst = perm[:count].astype(np.int32), perm[count:2 * count].astype(np.int32)
    src[::5], dst[2::7] = -1, blocks + 3
    ok = (src >= 0) & (dst < blocks)
    raw = lambda c: [x.view(torch.uint8).cpu().numpy().reshape(c.num_blocks, -1).copy() for x in (c.k, c.v, c.scales) if x is not None]  # noqa: E731
    want, want_other = raw(c), raw(other)
    to = rng.permutation(count + 9)[:count].astype(np.int32)
    for x, y in zip(want, want_other):
        y[to[src >= 0]] = x[src[src >= 0]]
        x[dst[ok]] = x[src[ok]]
    pk.kv_cache_copy(c, dev(src), dev(to), to=other)
    pk.kv_cache_copy(c, dev(src), dev(dst))
    torch.cuda.synchronize()
    for x, y in zip(raw(c) + raw(other), want + want_other):
        assert np.array_equal(x, y)


def test_copies_behind_four_gib():
    c = pk.new_kv_cache(70000, 32, 8, 128, pk.PK_BF16)             # 4.6 GB of keys
    c.k[69999], c.v[69999] = 3.0, 4.0
    pk.kv_cache_copy(c, dev([69999, 5]), dev([66666, 69998]))
    torch.cuda.synchronize()
    assert (c.k[66666] == 3).all() and (c.v[66666] == 4).all() and not c.k[69998].any() and not c.k[66667].any() and (c.k[69999] == 3).all()


def test_a_captured_step_and_another_stream():
    """Forking, reserving and copying replay from a graph while the lengths and what comes from what change."""
    rng, page, n, most, blocks = np.random.default_rng(8), 16, 12, 8, 200
    b = Batch(rng, n, most, blocks, page, 100)
    cache = pk.new_kv_cache(blocks, page, 2, 64, pk.PK_F8)
    cache.k.view(torch.uint8).copy_(torch.randint(0, 120, cache.k.shape, device=DEV, dtype=torch.uint8))
    state = [dev(b.table), dev(b.lens), dev(b.pages)]
    new = [torch.zeros_like(x) for x in state]
    refs, rows, grow = dev(b.refs), dev(np.arange(n)), dev(np.ones(n))
    served, src, dst = (dev(np.zeros(n)) for _ in range(3))
    ws = pk.new_pages_workspace(blocks)

    def step():
        pk.kv_pages_select(*state, rows, *new, refs, page)
        pk.kv_pages_reserve(*new, grow, refs, page, served, src, dst, ws)
        pk.kv_cache_copy(cache, src, dst)
        for x, y in zip(state, new):
            x.copy_(y)

    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            step()
    torch.cuda.current_stream().wait_stream(s)
    for turn in range(5):
        take, more = rng.integers(0, n, n).astype(np.int32), rng.integers(0, 4, n).astype(np.int32)
        rows.copy_(dev(take)), grow.copy_(dev(more))
        graph.replay()
        fresh = np.zeros((n, most), np.int32) if turn == 0 else b.table.copy()
        b.lens, b.pages = ob.pages_select(b.table, b.lens, b.pages, take, fresh, b.refs, page)
        b.table = fresh
        want = ob.pages_reserve(b.table, b.lens, b.pages, more, b.refs, page)
        got = host(*state, refs, served, src, dst)
        for g, w in zip(got, (b.table, b.lens, b.pages, b.refs) + want):
            assert np.array_equal(g, w)
        held = torch.arange(n, device=DEV)
        assert (held >= 0).all()                                   # (eager work in between)
        b.lens = np.minimum(b.lens + want[0] * more, b.pages * page).astype(np.int32)
        state[1].copy_(dev(b.lens))
