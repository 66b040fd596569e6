"""Attention over a paged cache whose values are ordinary but rarely drawn: rows of zeros, the smallest and the largest scales.

Tolerances are those of test_gpu_cache_step.py: 2^-8 (sum p |v| + |o|) + 1e-4 sum p |v| for the probabilities' rounding to bf16, and 2^-8 |o| for bf16
output.  Nothing in them depends on the scales of V, which are powers of two."""
import numpy as np
import pytest
import torch

from paper_2602_06072_amd import binding as pk
from tests import test_gpu_cache_paths as paths
from tests import test_gpu_cache_step as step

pytestmark = pytest.mark.gpu
DEV = "cuda"
ROWS = [(4, 1), (5, 4), (32, 1), (33, 1), (64, 1), (8, 8)]         # drafted tokens, query heads of a KV head


def one_request(seed, keys, drafts, heads, d, cache=pk.PK_F8, Hkv=2):
    s = step.make(seed, [keys - drafts], [drafts], heads * Hkv, Hkv, d, 16, cache)
    s["at"] = torch.from_numpy(s["slots"][0]).to(DEV)
    return s


def rows_of(s, seed, outstanding=None, score=10.0):
    """K and V of all the request's tokens: scores of N(0, 1), those of the outstanding keys `score`, and rows of V of N(0, 1)."""
    L, Hkv, d = len(s["at"]), s["c"].Hkv, s["c"].d
    g = step.gen(seed)
    k, v = (torch.randn(L, Hkv, d, generator=g, device=DEV) for _ in "kv")
    s["q"][..., 0] = 8.0
    k[..., 0] = 0.0
    if outstanding is not None:
        k[outstanding] = 0.0
        k[outstanding, :, 0] = score * d ** 0.5 / 8
    return k, v


def bytes_of(s, of_v):
    """(scale bytes of K or V, token by token) to be read, and a function that puts them."""
    x, at, page = s["c"].scales.view(torch.uint8), s["at"], s["c"].page_size

    def put(tokens, value):
        x[at[tokens] // page, :, of_v, at[tokens] % page] = value
    return put


@pytest.mark.parametrize("outstanding, score", [(None, 0.0), (301, 10.0), (slice(5, None, 32), 6.0)])        # (one of every 32: every wave has some)
@pytest.mark.parametrize("keys", [1000, 16000])
@pytest.mark.parametrize("drafts, heads", ROWS)
@pytest.mark.parametrize("d", [64, 128])
def test_rows_of_v_that_are_zero_keep_their_weight(drafts, heads, keys, outstanding, score, d):
    s = one_request(keys + drafts, keys, drafts, heads, d)
    k, v = rows_of(s, d, outstanding, score)
    zero = torch.rand(keys, generator=step.gen(1), device=DEV) < 0.5
    if outstanding is not None:
        zero[outstanding] = False
    v[zero] = 0.0
    pk.kv_cache_write(s["c"], k, v, s["at"])
    paths.dense(s, None, step.call(s, None))


@pytest.mark.parametrize("drafts, heads", [(2, 8), (2, 16), (7, 8)])
@pytest.mark.parametrize("d", [64, 128])
def test_zero_rows_in_many_short_requests(drafts, heads, d):
    """Tables of 256 keys and fewer, more requests than workgroups run at once: 16, 32 and 56 rows."""
    n = 300
    s = step.make(n + drafts, [150 + i % 50 for i in range(n)], [drafts] * n, 2 * heads, 2, d, 16, pk.PK_F8)
    at = torch.from_numpy(np.concatenate(s["slots"])).to(DEV)
    g = step.gen(d)
    k, v = (torch.randn(len(at), 2, d, generator=g, device=DEV) for _ in "kv")
    s["q"] *= 2                                                    # (scores of N(0, 4): some probabilities are below 2^-8)
    v[torch.rand(len(at), generator=g, device=DEV) < 0.5] = 0.0
    pk.kv_cache_write(s["c"], k, v, at)
    paths.dense(s, None, step.call(s, None))


@pytest.mark.parametrize("byte", [1, 2, 20, 254])
@pytest.mark.parametrize("drafts, heads", ROWS)
@pytest.mark.parametrize("d", [64, 128])
def test_smallest_and_largest_scales_of_v_beside_others(drafts, heads, byte, d):
    s = one_request(drafts + byte, 1000, drafts, heads, d)
    k, v = rows_of(s, d, 301)
    pk.kv_cache_write(s["c"], k, v, s["at"])
    some = torch.nonzero(torch.rand(1000, generator=step.gen(2), device=DEV) < 0.5)[:, 0]
    bytes_of(s, 1)(some, byte)
    if byte == 254:                                                # codes below 2^-6: sums of many stay below 2^127
        page = s["c"].page_size
        codes, blk, off = s["c"].v.view(torch.uint8), s["at"][some] // page, s["at"][some] % page
        codes[blk, :, off // 4, :, off % 4] &= 0x87
    paths.dense(s, None, step.call(s, None, torch.float32))


@pytest.mark.parametrize("drafts, heads", ROWS)
@pytest.mark.parametrize("d", [64, 128])
def test_all_of_v_with_the_smallest_scale(drafts, heads, d):
    """Values of some 2^-118: what comes out has to be right relative to them.  (Codes below 1, whose values are bf16 denormals, are at
    most 2^-8 of the rows' largest, and there are few.)"""
    s = one_request(drafts, 700, drafts, heads, d)
    k, v = rows_of(s, d)
    pk.kv_cache_write(s["c"], k, v, s["at"])
    bytes_of(s, 1)(slice(None), 1)
    out = step.call(s, None, torch.float32).double() * 2.0 ** 126
    bytes_of(s, 1)(slice(None), 127)
    paths.dense(s, None, out)


@pytest.mark.parametrize("drafts, heads", ROWS)
def test_the_smallest_scale_of_k(drafts, heads):
    """Keys of next to nothing: their scores are zero."""
    s = one_request(drafts, 700, drafts, heads, 128)
    k, v = rows_of(s, 5, 301)
    pk.kv_cache_write(s["c"], k, v, s["at"])
    bytes_of(s, 0)(torch.arange(0, 700, 3, device=DEV), 1)
    paths.dense(s, None, step.call(s, None))


@pytest.mark.parametrize("first, last", [(0, 32), (0, 64), (64, 700), (0, 1490)])
@pytest.mark.parametrize("drafts, heads", ROWS + [(17, 8)])
@pytest.mark.parametrize("d", [64, 128])
def test_keys_whose_scores_are_minus_infinity_have_no_weight(drafts, heads, first, last, d):
    """Infinite keys of a bf16 cache, at the front and where pieces begin; the others' results are finite."""
    s = one_request(drafts, 1500 + drafts, drafts, heads, d, pk.PK_BF16)
    k, v = rows_of(s, d)
    k[first:last, :, 0] = -float("inf")
    pk.kv_cache_write(s["c"], k, v, s["at"])
    paths.dense(s, None, step.call(s, None))


@pytest.mark.parametrize("keys, slope", [(300, 0.2), (600, 0.09), (1500, 0.03), (300, -0.2), (64, 0.9), (64, -0.9)])
@pytest.mark.parametrize("cache", [pk.PK_F8, pk.PK_BF16])
@pytest.mark.parametrize("drafts, heads", ROWS + [(17, 8)])
@pytest.mark.parametrize("d", [64, 128])
def test_scores_that_rise_and_fall_from_tile_to_tile(drafts, heads, cache, keys, slope, d):
    """Scores up to 60 that change by less and by more than 2^8 from one half-tile of 32 keys to the next, in the order of the keys.  fp32
    sums of four products at a time err by 60 * 2^-24 each, 32 of them at most, half of it one way: 6e-5 of the 1e-4 that there are."""
    s = one_request(drafts + keys, keys, drafts, heads, d, cache)
    k, v = rows_of(s, d)
    ramp = slope * torch.arange(keys, device=DEV)
    k[..., 0] = ((ramp - ramp.mean()) * d ** 0.5 / 8)[:, None]
    pk.kv_cache_write(s["c"], k, v, s["at"])
    paths.dense(s, None, step.call(s, None))
