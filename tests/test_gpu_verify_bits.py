"""Judging of drafted tokens next to borders that only 64 bits tell apart: probabilities of two tokens whose ratio is so near to a random number
that an error of 1e-13 falls to the other side.

A row has logits 0 and x (others are -inf), |x| <= 3: the weights are 1 and e^x.  In 64 bits x / ln 2 is off by 2^-53 of itself twice (the factor's
rounding and the product's), at most 4.4 * 2 * 1.2e-16 * ln 2 = 7e-16 of the weight; the exponential by 4e-16, and sums, quotients and products by 1.2e-16 each, of which there are up to eight:
together below 3e-15.  The cases here are 1e-14 to 3e-13 off their border, found with 64 bits of fraction (1e-19)."""
import numpy as np
import pytest
import torch

from tests.test_gpu_verify import call, check

pytestmark = pytest.mark.gpu
LEAST, MOST = 1e-14, 3e-13
VOCAB = 40
real = np.longdouble


def near_borders(rng, value, count, tries=1 << 20):
    """(x, y, u, above): logits x and y in fp32, u in fp32 and whether value(x, y) > u, for `count` values that are next to a number u of fp32."""
    got = []
    while sum(len(g[0]) for g in got) < count:
        x, y = (rng.uniform(-3, 3, tries).astype(np.float32) for _ in "xy")
        v = value(np.exp(x.astype(real)), np.exp(y.astype(real)))
        u = v.astype(np.float32)
        off = (v - u.astype(real)) / v
        hit = (np.abs(off) > LEAST) & (np.abs(off) < MOST) & (u < 1)
        got.append((x[hit], y[hit], u[hit], off[hit] > 0))
    return [np.concatenate(z)[:count] for z in zip(*got)]


def rows(rng, x, tokens):
    """Rows with 0 at a place, x at a later one; their places."""
    places = np.sort(np.stack([rng.permutation(VOCAB)[:2] for _ in x]), 1)
    r = np.full((len(x), tokens, VOCAB), -np.inf, np.float32)
    return r, places


@pytest.mark.parametrize("seed", range(3))
def test_draws_next_to_a_border(seed):
    """The first token is drawn if 1 > u (1 + e^x)."""
    rng = np.random.default_rng(seed)
    x, _, u, first = near_borders(rng, lambda e, _: 1 / (1 + e), 60)
    r, places = rows(rng, x, 1)
    n = len(x)
    r[np.arange(n), 0, places[:, 0]], r[np.arange(n), 0, places[:, 1]] = 0, x
    s = dict(target=torch.from_numpy(r[:, 0]), draft=None, vocab=VOCAB, tokens=np.zeros(n, np.int32), q_start=np.arange(n + 1, dtype=np.int32), sizes=[1] * n, mask=None,
             temperature=None, accept=np.zeros(n, np.float32), sample=u, max_q=1)
    got = call(s)
    assert np.array_equal(got[2], np.where(first, places[:, 0], places[:, 1]))
    assert 5 < first.sum() < 55
    check(s, got)


@pytest.mark.parametrize("drawn, tree", [(True, True), (True, False), (False, True)])
@pytest.mark.parametrize("seed", range(2))
def test_choices_next_to_a_border(drawn, tree, seed):
    """The second token's one child, the token of logit 0, stays if P > u Q, or without draft logits P > u."""
    rng = np.random.default_rng(10 + seed)
    value = (lambda e, f: (1 + f) / (1 + e)) if drawn else (lambda e, _: 1 / (1 + e))
    x, y, u, stays = near_borders(rng, value, 60)
    r, places = rows(rng, x, 2)
    n = len(x)
    target, draft = r, r.copy()
    for t in range(2):
        target[np.arange(n), t, places[:, 0]], target[np.arange(n), t, places[:, 1]] = 0, x
        draft[np.arange(n), t, places[:, 0]], draft[np.arange(n), t, places[:, 1]] = 0, y
    accept, tokens = np.zeros((n, 2), np.float32), np.zeros((n, 2), np.int32)
    accept[:, 1], tokens[:, 1] = u, places[:, 0]
    flat = lambda z: torch.from_numpy(z.reshape(2 * n, VOCAB))  # noqa: E731
    s = dict(target=flat(target), draft=flat(draft) if drawn else None, vocab=VOCAB, tokens=tokens.reshape(-1), q_start=np.arange(0, 2 * n + 1, 2, dtype=np.int32), sizes=[2] * n,
             mask=np.tile(np.array([1, 3], np.uint64), n) if tree else None, temperature=None, accept=accept.reshape(-1), sample=np.full(n, 0.5, np.float32), max_q=2)
    got = call(s)
    assert np.array_equal(got[1] == 2, stays)
    assert 5 < stays.sum() < 55
