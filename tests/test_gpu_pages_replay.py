"""Replays of captured steps on the pages of a batch: tables, counts, lists and every byte of the caches against oracle/branch.py, with eager work between the replays."""
import numpy as np
import pytest
import torch

from oracle import branch as ob
from paper_2602_06072_amd import binding as pk
from tests.test_gpu_pages import Batch, dev, host

pytestmark = pytest.mark.gpu
DEV = "cuda"


def parts(c):
    return [x for x in (c.k, c.v, c.scales) if x is not None]


def raw(c):
    torch.cuda.synchronize()
    return [x.view(torch.uint8).cpu().numpy().reshape(c.num_blocks, -1).copy() for x in parts(c)]


@pytest.mark.parametrize("n, most, blocks", [(12, 8, 200), (1300, 3, 6000)])
def test_copies_follow_the_lists_of_every_replay(n, most, blocks):
    """Forks, pages for new tokens and the copies of two layers' caches, one of 8 bits and one of bf16."""
    rng, page, g = np.random.default_rng(n), 16, torch.Generator(device=DEV).manual_seed(n)
    b = Batch(rng, n, most, blocks, page, 16 * most - 20)
    caches = [pk.new_kv_cache(blocks, page, 2, 64, t) for t in (pk.PK_F8, pk.PK_BF16)]
    for c in caches:
        for x in parts(c):
            y = x.view(torch.uint8).view(-1)
            y.copy_(torch.randint(0, 256, y.shape, generator=g, device=DEV, dtype=torch.uint8))
    want_bytes = [raw(c) for c in caches]
    state = [dev(b.table), dev(b.lens), dev(b.pages)]
    new = [torch.zeros_like(x) for x in state]
    refs, rows, grow = dev(b.refs), dev(np.arange(n)), dev(np.ones(n))
    served, src, dst = (dev(np.zeros(n)) for _ in range(3))
    ws = pk.new_pages_workspace(blocks)

    def step():
        pk.kv_pages_select(*state, rows, *new, refs, page)
        pk.kv_pages_reserve(*new, grow, refs, page, served, src, dst, ws)
        for c in caches:
            pk.kv_cache_copy(c, src, dst)
        for x, y in zip(state, new):
            x.copy_(y)

    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    copies = 0
    for turn in range(5):
        take, more = rng.integers(0, n, n).astype(np.int32), rng.integers(0, 4, n).astype(np.int32)
        rows.copy_(dev(take)), grow.copy_(dev(more))
        graph.replay()
        fresh = np.zeros((n, most), np.int32) if turn == 0 else b.table.copy()
        b.lens, b.pages = ob.pages_select(b.table, b.lens, b.pages, take, fresh, b.refs, page)
        b.table = fresh
        want = ob.pages_reserve(b.table, b.lens, b.pages, more, b.refs, page)
        for x, y in zip(host(*state, refs, served, src, dst), (b.table, b.lens, b.pages, b.refs) + want):
            assert np.array_equal(x, y)
        for i in np.nonzero(want[1] >= 0)[0]:
            for layer in want_bytes:
                for x in layer:
                    x[want[2][i]] = x[want[1][i]]
            copies += 1
        for c, layer in zip(caches, want_bytes):
            for x, y in zip(raw(c), layer):
                assert np.array_equal(x, y)
        b.lens = np.minimum(b.lens + want[0] * more, b.pages * page).astype(np.int32)
        state[1].copy_(dev(b.lens))
        k, v = (torch.randn(3, 2, 64, generator=g, device=DEV) for _ in "kv")              # eager writes in between, into places of request 0
        if b.lens[0] >= 3:
            slots = dev(b.table[0, np.arange(3) // page] * page + np.arange(3) % page).long()
            for c, layer in zip(caches, want_bytes):
                pk.kv_cache_write(c, k, v, slots)
                layer[:] = raw(c)
    assert copies > 5


def test_compaction_replays():
    rng, page, blocks, n = np.random.default_rng(3), 16, 3000, 40
    g = torch.Generator(device=DEV).manual_seed(3)
    c = pk.new_kv_cache(blocks, page, 1, 64, pk.PK_F8)
    for x in parts(c):
        y = x.view(torch.uint8).view(-1)
        y.copy_(torch.randint(0, 256, y.shape, generator=g, device=DEV, dtype=torch.uint8))
    table, pages, refs = dev(np.zeros((n, 30))), dev(np.zeros(n)), dev(np.zeros(blocks))
    new_refs, src, dst = torch.zeros_like(refs), dev(np.zeros(700)), dev(np.zeros(700))
    ws = pk.new_pages_workspace(blocks)

    def step():
        pk.kv_pages_compact(table, pages, refs, table, new_refs, src, dst, ws)
        pk.kv_cache_copy(c, src, dst)

    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for turn in range(4):
        b = Batch(rng, n, 30, blocks, page, 100 + 100 * turn)
        for x, y in ((table, b.table), (pages, b.pages), (refs, b.refs)):
            x.copy_(dev(y))
        bytes_before = raw(c)
        graph.replay()
        want = ob.pages_compact(b.table, b.pages, b.refs, 700)
        for x, y in zip(host(table, new_refs, src, dst), want):
            assert np.array_equal(x, y)
        for x, y in zip(raw(c), bytes_before):
            moved = want[2] >= 0
            y[want[3][moved]] = y[want[2][moved]]
            assert np.array_equal(x, y)
