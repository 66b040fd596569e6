"""The workspace of the judging of drafted tokens: one of the largest batch serves all smaller ones (sizes can be asked for without a GPU)."""
import random

import pytest

from paper_2602_06072_amd import binding as pk


def size(n, total_q, vocab):
    return pk.lib().pk_draft_verify_workspace_bytes(n, total_q, vocab)


@pytest.mark.parametrize("vocab", [1, 4096, 4097, 32000, 50257, 128256, 151936, 262144, 262145, 1 << 26])
def test_the_size_does_not_fall_with_the_batch(vocab):
    by_tokens = [size(4, t, vocab) for t in range(0, 4200)]
    assert by_tokens == sorted(by_tokens)
    by_requests = [size(n, 100, vocab) for n in range(0, 700)]
    assert by_requests == sorted(by_requests)
    for t in (1, 5, 8, 16):                                        # of as many tokens each
        together = [size(n, n * t, vocab) for n in range(1, 2200)]
        assert together == sorted(together)


def test_the_size_does_not_fall_with_the_vocabulary():
    for n, t in ((1, 1), (3, 64), (64, 640), (300, 2100)):
        sizes = [size(n, t, v) for v in [*range(1, 12000, 7), *range(250000, 280000, 97), *range(1 << 20, 1 << 26, 65537), 1 << 26]]
        assert sizes == sorted(sizes)


def test_the_size_is_enough_for_any_smaller_batch():
    rng = random.Random(5)
    for _ in range(20000):
        n, t, v = (int(2 ** rng.uniform(0, x)) for x in (16, 20, 26))
        n = min(n, 65535)
        assert size(rng.randint(0, n), rng.randint(0, t), rng.randint(1, v)) <= size(n, t, v)


def test_the_size_stays_a_small_part_of_the_logits():
    """As said beside the sizes: no more than 2 * 16 bytes for every piece of up to 2048 + total_q, 256 spans of 16 bytes a request, and some for each token."""
    for n, t, v in ((1, 1, 128256), (64, 640, 128256), (256, 2048, 32000), (2000, 16000, 151936)):
        assert 0 < size(n, t, v) <= 65536 * 4 + 32 * (2048 + t) + 4096 * n + 160 * t + 1024
