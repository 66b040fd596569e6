"""Outputs and a workspace of the judging of drafted tokens that lie in rows of logits are refused before anything is launched (no GPU involved)."""
import pytest

from paper_2602_06072_amd import binding as pk
from tests.test_branch_refusals import EINVAL, M, P, refused, verify

ROWS = 12 * 1000 * 2                        # bytes of 12 rows of 1000 logits


@pytest.mark.parametrize("change, word", [
    (dict(keep=P), "keep overlaps target"), (dict(keep=P + ROWS - 4), "keep overlaps target"), (dict(keep=P - 44), "keep overlaps target"), (dict(count=P + 12000), "keep_count overlaps target"),
    (dict(after=P + 20), "next_token overlaps target"), (dict(after=P + M), "next_token overlaps draft"), (dict(keep=P + M + ROWS - 8), "keep overlaps draft"),
    (dict(ws=P + 256), "workspace overlaps target"), (dict(ws=P + M + 256), "workspace overlaps draft"), (dict(ws=P - 256), "workspace overlaps target"),
    (dict(ts=1500, keep=P + 3000), "keep overlaps target"), (dict(ts=1500, keep=P + 2960), "keep overlaps target"), (dict(ts=1500, count=P + 11 * 3000 + 1996), "keep_count overlaps target"),
    (dict(ds=1100, count=P + M + 2196), "keep_count overlaps draft"), (dict(dtype=pk.PK_F32, keep=P + 2 * ROWS - 4), "keep overlaps target"),
    (dict(total=1, ts=0, draft=None, after=P + 1996), "next_token overlaps target")])
def test_outputs_in_rows_of_logits(change, word):
    refused(verify(**change), EINVAL, word)
