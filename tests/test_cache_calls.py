"""How the calls of the paged cache take their arguments, without a GPU: calls of no requests reach the library and return."""
import pytest
import torch

from paper_2602_06072_amd import binding as pk


def empty_keep(n=0):
    i32 = lambda *shape: torch.zeros(*shape, dtype=torch.int32)  # noqa: E731
    c = pk.new_kv_cache(4, 16, 2, 64, device="cpu")
    return (c, i32(n, 3), i32(n), i32(n + 1)), (i32(n, 5), i32(n), i32(n))


class Stream:
    cuda_stream = 0


def test_keep_takes_the_bound_of_the_drafted_tokens_or_not():
    where, what = empty_keep()
    for args in (what, (5, *what), (0, *what), (64, *what)):
        assert pk.kv_cache_keep(*where, *args, stream=Stream) is what[2]
        assert pk.kv_cache_keep(*where, *args, Stream) is what[2]
    assert pk.kv_cache_keep(*where, keep=what[0], keep_count=what[1], new_lens=what[2], stream=Stream) is what[2]
    for args in ((5, *what[:2]), (-1, *what), (65, *what), (5, *what, Stream, Stream), (*what, Stream, Stream)):
        with pytest.raises(pk.PackInferError):
            pk.kv_cache_keep(*where, *args)
