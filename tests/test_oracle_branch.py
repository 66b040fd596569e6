"""Pins of oracle/branch.py: judged drafts are distributed as the target says (enumerated, not drawn), pages are handed out
as worked by hand."""
import itertools

import numpy as np
import pytest

from oracle import branch as ob


def distribution(P, Q, kids, drawn):
    """Distribution of the token behind token 0 with `kids` drafted ones, by enumeration: the drafted tokens over what they are drawn
    from, u over the middles of a fine grid, sampling over a grid too."""
    V, out = len(P), np.zeros(len(P))
    target = np.log(np.stack([P] * (kids + 1)))
    draft = np.log(np.stack([Q] * (kids + 1))) if drawn else None
    mask = [1] + [1 | 2 << t for t in range(kids)]
    grid = (np.arange(40) + 0.5) / 40
    for tokens in itertools.product(range(V), repeat=kids):
        weight = np.prod([Q[x] for x in tokens]) if drawn else V ** -kids
        for us in itertools.product(grid[::2] if kids > 1 else grid, repeat=kids):
            kept, _ = ob.draft_verify(target, draft, (0,) + tokens, mask, 1.0, (0.0,) + us, 0.5, 9)
            w = weight / len(grid[::2] if kids > 1 else grid) ** kids
            if len(kept) == 2:
                out[tokens[kept[1] - 1]] += w
            else:
                for s in grid:
                    out[ob.draft_verify(target, draft, (0,) + tokens, mask, 1.0, (0.0,) + us, s, 9)[1]] += w / len(grid)
    return out


@pytest.mark.parametrize("kids, drawn", [(1, True), (2, True), (1, False), (2, False)])
def test_the_next_token_is_distributed_as_the_target(kids, drawn):
    P, Q = np.array([0.5, 0.2, 0.3]), np.array([0.25, 0.6, 0.15])
    # grids of 20 and 40 points: each acceptance and each draw is off by half a step of 1/20 and 1/40 at most
    assert np.abs(distribution(P, Q, kids, drawn) - P).max() < kids * 0.025 + 0.0125


def test_judging_by_hand():
    t = np.log(np.array([[0.1, 0.6, 0.3], [0.2, 0.2, 0.6], [0.3, 0.3, 0.4]]))
    q = np.log(np.array([[0.5, 0.3, 0.2], [0.2, 0.7, 0.1], [1 / 3] * 3]))
    # token 1 stays: 0.6 > 0.9 * 0.3; token 2: 0.2 > 0.25 * 0.7; behind it 0.65 of (0.3, 0.6, 1)
    assert ob.draft_verify(t, q, [0, 1, 1], None, 1.0, [0, 0.9, 0.25], 0.65, 9) == ([0, 1, 2], 2)
    # token 1 does not: 0.1 < 0.3 * 0.5; residual (0, 0.3, 0.1): 0.74 falls into token 1, 0.76 into token 2
    assert ob.draft_verify(t, q, [0, 0, 1], None, 1.0, [0, 0.3, 0.0], 0.74, 9) == ([0], 1)
    assert ob.draft_verify(t, q, [0, 0, 1], None, 1.0, [0, 0.3, 0.0], 0.76, 9) == ([0], 2)
    # siblings without draft: 0 goes (0.1 < 0.2), then 0.6 of 0.9 against 0.7: it goes too, 2 is left
    assert ob.draft_verify(t, None, [0, 0, 1], [1, 3, 5], 1.0, [0, 0.2, 0.7], 0.3, 9) == ([0], 2)
    assert ob.draft_verify(t, None, [0, 0, 1], [1, 3, 5], 1.0, [0, 0.2, 0.6], 0.29, 9) == ([0, 2], 0)
    assert ob.draft_verify(t, q, [0, 1, 2], None, 0.0, [0, 0.99, 0.99], 0.9, 9) == ([0, 1, 2], 2)
    assert ob.draft_verify(t, q, [0, 1, 2], None, 0.0, [0, 0.99, 0.99], 0.9, 2) == ([0, 1], 2)
    assert ob.draft_verify(np.full((1, 3), -np.inf), None, [0], None, 1.0, [0], 0.5, 9) == ([0], -1)


def test_pages_by_hand():
    table = np.array([[4, 2, 0], [5, 0, 0]], np.int32)
    lens, pages, refs = np.array([18, 16], np.int32), np.array([2, 1], np.int32), np.array([0, 0, 1, 0, 1, 1], np.int32)
    new = np.zeros((3, 3), np.int32)
    ls, ps = ob.pages_select(table, lens, pages, [0, 0, 7], new, refs, 16)
    assert new.tolist() == [[4, 2, 0], [4, 2, 0], [0, 0, 0]] and ls.tolist() == [18, 18, 0] and ps.tolist() == [2, 2, 0]
    assert refs.tolist() == [0, 0, 2, 0, 2, 0]
    served, src, dst = ob.pages_reserve(new, ls, ps, np.array([1, 15, 40], np.int32), refs, 16)
    # request 0 leaves block 2 to request 1 and gets block 0; request 1 grows into block 1; request 2 gets 3 and 5, and no third one
    assert served.tolist() == [1, 1, 0] and src.tolist() == [2, -1, -1] and dst.tolist() == [0, -1, -1]
    assert new.tolist() == [[4, 0, 0], [4, 2, 1], [0, 0, 0]] and ps.tolist() == [2, 3, 0] and refs.tolist() == [1, 1, 1, 0, 2, 0]
    refs = np.array([0, 3, 0, 0, 2, 1], np.int32)
    table = np.array([[5, 4], [1, 4]], np.int32)
    nt, nr, src, dst = ob.pages_compact(table, np.array([2, 1]), refs, 3)
    assert src.tolist() == [4, 5, -1] and dst.tolist() == [0, 2, -1] and nt.tolist() == [[2, 0], [1, 4]] and nr.tolist() == [2, 3, 1, 0, 0, 0]
