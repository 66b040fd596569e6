"""One workspace of the attention of drafted tokens for calls of different sizes: each result is that with a workspace of its own, bit for bit."""
import pytest
import torch

from paper_2602_06072_amd import binding as pk
from tests import test_gpu_cache_paths as paths
from tests import test_gpu_cache_step as step

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("cache", [pk.PK_F8, pk.PK_BF16])
@pytest.mark.parametrize("Hkv, d", [(8, 128), (2, 64)])
def test_a_workspace_made_for_few_long_drafts_serves_many_single_tokens(Hkv, d, cache):
    """Partial results of 128 rows lie where the small calls have nothing; theirs are counted where nobody else writes."""
    calls = [([3000 + 500 * i for i in range(8)], [64] * 8, 2), ([40 + 37 * i for i in range(200)], [1] * 200, 2), ([9000, 4, 700], [2, 1, 3], 4),
             ([5000 - 90 * i for i in range(50)], [3] * 50, 8), ([6000], [1], 1)]
    made = [step.make(17 + i, ctx, drafts, heads * Hkv, Hkv, d, 16, cache) for i, (ctx, drafts, heads) in enumerate(calls)]
    own = [step.call(s, None) for s in made]
    paths.dense(made[1], None, own[1])
    sizes = [int(pk.lib().pk_tree_attn_workspace_bytes(len(s["lens"]), s["max_q"], s["q"].shape[1], Hkv, d)) for s in made]
    assert max(sizes) == sizes[0]
    ws = torch.zeros(sizes[0], dtype=torch.uint8, device="cuda")   # as for the first of them
    for i in (0, 1, 2, 0, 3, 1, 4, 0, 1, 3, 2):
        assert torch.equal(step.call(made[i], None, ws=ws), own[i]), i
