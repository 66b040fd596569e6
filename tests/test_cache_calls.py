"""How the calls of the paged cache take their arguments, without a GPU: calls of no requests reach the library and return."""
import pytest
import torch

from paper_2602_06072_amd import binding as pk
from tests.test_cache_refusals import cache, refused, rope, rows

EINVAL, P = -1, 1 << 20


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


def test_a_new_cache_holds_rows_of_zeros_as_the_format_has_them():
    c = pk.new_kv_cache(3, 32, 2, 64, device="cpu")
    assert (c.k.view(torch.uint8) == 0).all() and (c.v.view(torch.uint8) == 0).all()
    assert (c.scales.view(torch.uint8) == 1).all()                 # 2^-126, the smallest scale: byte 0 stands for none
    b = pk.new_kv_cache(3, 32, 2, 64, pk.PK_BF16, device="cpu")
    assert b.scales is None and (b.k == 0).all() and (b.v == 0).all()


@pytest.mark.parametrize("Hq, Hkv, d", [(32, 8, 128), (16, 1, 64), (64, 64, 64), (2048, 1024, 128)])
def test_the_counts_of_a_workspace_do_not_grow_with_requests(Hq, Hkv, d):
    """What has to be zero lies at the front and is as long for every call: more requests take the eight bytes that each call writes before it reads them."""
    size = pk.lib().pk_tree_attn_workspace_bytes
    for max_q in (1, 5, 64):
        assert size(65535, max_q, Hq, Hkv, d) - size(1, max_q, Hq, Hkv, d) == 65535 * 8 // 256 * 256
    assert size(1, 64, Hq, Hkv, d) >= size(1, 1, Hq, Hkv, d) > 0


@pytest.mark.parametrize("tokens, ts, hs", [((1 << 31) - 1, 1 << 29, 128), (1 << 20, 1 << 40, 128), (4, 1 << 58, 128), (1, 1 << 62, 128), (4, 4096, 1 << 57)])
def test_strides_whose_products_leave_64_bits_are_refused(tokens, ts, hs):
    far, near = rows(ts=ts, hs=hs), rows(ts=4096)
    L = pk.lib()
    for q, k, q_out, k_out in ((far, near, near, near), (near, far, near, near), (near, near, far, near), (near, near, near, far)):
        refused(L.pk_qk_norm_rope(q, k, q_out, k_out, None, None, 0.0, None, tokens, 8, 8, 128, None), EINVAL, "stride out of range")
    refused(L.pk_kv_cache_write(cache(), rows(), far, P, tokens, None), EINVAL, "stride out of range")
    refused(L.pk_kv_cache_read(cache(), P, 4, P, P, 3, near, far, tokens, None), EINVAL, "stride out of range")


def test_strides_are_accepted_up_to_the_bound():
    """The next argument is refused: the strides were not."""
    L, most = pk.lib(), (1 << 59) // ((1 << 31) - 1) // 8 * 8
    for ts, hs, tokens in ((most, 1 << 56, (1 << 31) - 1), (1 << 59, 128, 1), (1 << 40, 1 << 41, 1 << 19)):
        far = rows(ts=ts, hs=hs)
        refused(L.pk_qk_norm_rope(far, far, None, None, None, None, 0.0, None, tokens, 8, 8, 128, None), EINVAL, "q_out is NULL")


@pytest.mark.parametrize("stride, axes", [(1 << 62, 3), ((1 << 59) + 4, 1), ((1 << 63) - 1, 255)])
def test_axis_strides_whose_products_leave_64_bits_are_refused(stride, axes):
    refused(pk.lib().pk_qk_norm_rope(rows(ts=4096), rows(), rows(ts=4096), rows(), None, None, 0.0, rope(stride=stride, axes=axes), 4, 32, 8, 128, None), EINVAL, "axis_stride")


@pytest.mark.parametrize("name, words", [("lens", 3), ("start", 4), ("count", 3), ("keep", 15), ("table", 12)])
def test_new_lengths_inside_of_an_array_that_is_read_are_refused(name, words):
    """3 requests, 5 kept tokens, 4 pages each: places in front of, in and behind every array."""
    at = dict(lens=P, start=P + 4096, count=P + 8192, keep=P + 12288, table=P + 16384)

    def keep(new, max_keep=5):
        return pk.lib().pk_kv_cache_keep(cache(), at["table"], 4, at["lens"], at["start"], 3, at["keep"], max_keep, at["count"], new, None)
    for word in (-2, 0, words - 1):
        refused(keep(at[name] + 4 * word), EINVAL, "new_lens must not be")
    if torch.cuda.is_available():
        return                                                     # (the others would be launched)
    for word in (-3, words):
        refused(keep(at[name] + 4 * word), -4, "")
    if name == "keep":
        refused(keep(at["keep"], 0), -4, "")                       # of no columns: nothing is read there


def test_batches_of_nothing_are_no_work_for_the_binding():
    """Tensors without elements, whose addresses are null: no tokens, no requests, tables without columns."""
    f = lambda *shape, dtype=torch.bfloat16: torch.zeros(*shape, dtype=dtype)  # noqa: E731
    i32 = lambda *shape: torch.zeros(*shape, dtype=torch.int32)  # noqa: E731
    c, q, k = pk.new_kv_cache(4, 16, 2, 64, device="cpu"), f(0, 8, 64), f(0, 2, 64)
    slots, rope = f(0, dtype=torch.int64), pk.Rope(f(4, 2, 32, dtype=torch.float32), i32(0))
    assert rope.positions.data_ptr() == 0
    w = f(64)
    assert pk.qk_norm_rope(q, k, q.clone(), k.clone(), w, w, 1e-6, rope, stream=Stream)
    assert pk.kv_cache_write(c, k, k, slots, stream=Stream) is c
    assert pk.qkv_cache_write(c, q, k, k, slots, q, w, w, 1e-6, rope, stream=Stream) is q
    for table in (i32(0, 3), i32(0, 0)):
        assert pk.kv_cache_read(c, table, i32(0), i32(0), k, k, stream=Stream)
        ws = pk.new_tree_workspace(0, 0, 8, 2, 64, device="cpu")
        assert pk.tree_attn(c, q, i32(1), 0, None, table, i32(0), q, 0.1, ws, stream=Stream) is q
        lens = i32(0)
        assert pk.kv_cache_keep(c, table, i32(0), i32(1), i32(0, 0), i32(0), lens, stream=Stream) is lens
    assert pk.tree_attn(c, q, i32(4), 5, f(0, dtype=torch.int64), i32(3, 2), i32(3), q, 0.1, ws, stream=Stream) is q     # requests without drafted tokens


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_strides_of_one_token_and_of_one_head_do_not_matter(dtype):
    base = torch.zeros(5, 3, 131, dtype=dtype)                     # rows of an odd number of columns
    one_token, one_head, one_row = base[2:3, :, :128], torch.zeros(5, 131 * 8, dtype=dtype)[:, None, :128].as_strided((5, 1, 128), (1048, 131, 1)), base[1:2, 1:2, :128]
    unpacked = lambda x: pk._ROWS.unpack(pk._rows(x, "x"))[1:3]  # noqa: E731
    assert unpacked(one_token) == (0, 131) and unpacked(one_head) == (1048, 0) and unpacked(one_row) == (0, 0)
    row = torch.empty_strided((1, 1, 128), (77, 5, 1), dtype=dtype).zero_()
    L, r = pk.lib(), pk._rows(row, "row")
    refused(L.pk_qk_norm_rope(r, r, r, None, None, None, 0.0, None, 1, 1, 1, 128, None), EINVAL, "k_out is NULL")      # (the others were accepted)
    far = rows(ts=77, hs=5)
    refused(L.pk_qk_norm_rope(far, r, r, r, None, None, 0.0, None, 1, 1, 1, 128, None), EINVAL, "multiples of 16 bytes")   # as the header says
