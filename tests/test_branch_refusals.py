"""What the calls of pages, shared attention and judging refuse: wrong arguments give a code and a message before anything is
launched (no GPU involved), and empty calls are no work."""
import pytest

from paper_2602_06072_amd import binding as pk

EINVAL, EUNSUPPORTED = -1, -3
P, M = 1 << 30, 1 << 28                     # addresses that are never read, M apart
NAN = float("nan")


def refused(rc, code, word):
    assert rc == code, (rc, pk.lib().pk_last_error())
    assert word in pk.lib().pk_last_error().decode(), pk.lib().pk_last_error()


def cache(k=P, v=P + M, scales=P + 2 * M, blocks=10, page=16, Hkv=8, d=128, dtype=pk.PK_F8):
    return pk._CACHE.pack(k, v, scales, blocks, page, Hkv, d, dtype)


SELECT = dict(table=P, lens=P + M, pages=P + 2 * M, n=4, most=8, rows=P + 3 * M, m=6, new_table=P + 4 * M, new_lens=P + 5 * M, new_pages=P + 6 * M, refs=P + 7 * M,
              blocks=100, page=16)


def select(**change):
    a = {**SELECT, **change}
    return pk.lib().pk_kv_pages_select(a["table"], a["lens"], a["pages"], a["n"], a["most"], a["rows"], a["m"], a["new_table"], a["new_lens"], a["new_pages"],
                                       a["refs"], a["blocks"], a["page"], None)


@pytest.mark.parametrize("change, word", [
    (dict(table=None), "block_table is NULL"), (dict(lens=None), "lens is NULL"), (dict(pages=None), "pages is NULL"), (dict(rows=None), "from is NULL"),
    (dict(new_table=None), "new_table is NULL"), (dict(new_lens=None), "new_lens is NULL"), (dict(new_pages=None), "new_pages is NULL"), (dict(refs=None), "refs is NULL"),
    (dict(n=-1), "n <"), (dict(m=-1), "n_new"), (dict(n=65536), "65536"), (dict(m=65536), "65536"), (dict(most=0), "max_blocks"), (dict(most=-1), "max_blocks"),
    (dict(most=1 << 28), "max_blocks"), (dict(blocks=0), "num_blocks"), (dict(blocks=1 << 31), "num_blocks"), (dict(page=0), "page_size"), (dict(lens=P + M + 2), "aligned"),
    (dict(new_table=P), "overlaps"), (dict(new_table=P + 4 * 8 * 4 - 4), "overlaps"), (dict(new_lens=P + M), "overlaps"), (dict(new_pages=P + 3 * M + 20), "overlaps"),
    (dict(refs=P + 4 * M), "overlaps"), (dict(new_pages=P + 5 * M), "overlaps"), (dict(refs=P + 2 * M - 396), "overlaps")])
def test_select_refuses(change, word):
    refused(select(**change), EINVAL, word)


RESERVE = dict(table=P, lens=P + M, pages=P + 2 * M, n=4, most=8, grow=P + 3 * M, refs=P + 4 * M, blocks=100, page=16, served=P + 5 * M, src=P + 6 * M,
               dst=P + 7 * M, ws=P + 8 * M, bytes=1 << 20)


def reserve(**change):
    a = {**RESERVE, **change}
    return pk.lib().pk_kv_pages_reserve(a["table"], a["lens"], a["pages"], a["n"], a["most"], a["grow"], a["refs"], a["blocks"], a["page"], a["served"], a["src"],
                                        a["dst"], a["ws"], a["bytes"], None)


@pytest.mark.parametrize("change, word", [
    (dict(table=None), "block_table is NULL"), (dict(lens=None), "lens is NULL"), (dict(pages=None), "pages is NULL"), (dict(grow=None), "grow is NULL"),
    (dict(refs=None), "refs is NULL"), (dict(served=None), "served is NULL"), (dict(src=None), "copy_src is NULL"), (dict(dst=None), "copy_dst is NULL"),
    (dict(ws=None), "workspace"), (dict(ws=P + 8 * M + 128), "workspace"), (dict(bytes=1023), "smaller"), (dict(n=-1), "n <"), (dict(most=0), "max_blocks"),
    (dict(blocks=-5), "num_blocks"), (dict(page=-16), "page_size"), (dict(dst=P + 6 * M), "overlaps"), (dict(grow=P + 5 * M), "overlaps"), (dict(lens=P + 2 * M), "overlaps"),
    (dict(refs=P + 8 * M), "overlaps"), (dict(refs=P + 8 * M + 16), "overlaps")])
def test_reserve_refuses(change, word):
    refused(reserve(**change), EINVAL, word)


COMPACT = dict(table=P, pages=P + M, n=4, most=8, refs=P + 2 * M, blocks=100, new_table=P + 3 * M, new_refs=P + 4 * M, src=P + 5 * M, dst=P + 6 * M, moves=50,
               ws=P + 7 * M, bytes=1 << 20)


def compact(**change):
    a = {**COMPACT, **change}
    return pk.lib().pk_kv_pages_compact(a["table"], a["pages"], a["n"], a["most"], a["refs"], a["blocks"], a["new_table"], a["new_refs"], a["src"], a["dst"],
                                        a["moves"], a["ws"], a["bytes"], None)


@pytest.mark.parametrize("change, word", [
    (dict(table=None), "block_table is NULL"), (dict(pages=None), "pages is NULL"), (dict(refs=None), "refs is NULL"), (dict(new_table=None), "new_table is NULL"),
    (dict(new_refs=None), "new_refs is NULL"), (dict(src=None), "copy_src is NULL"), (dict(dst=None), "copy_dst is NULL"), (dict(moves=-1), "max_moves"),
    (dict(new_refs=P + 2 * M), "overlaps"), (dict(new_table=P + 16), "overlaps"), (dict(dst=P + 5 * M + 4), "overlaps"), (dict(ws=None), "workspace"),
    (dict(bytes=0), "smaller"), (dict(n=1 << 20), "n <"), (dict(blocks=0), "num_blocks")])
def test_compact_refuses(change, word):
    refused(compact(**change), EINVAL, word)


@pytest.mark.parametrize("change, code, word", [
    (dict(f=None), EINVAL, "cache is NULL"), (dict(t=None), EINVAL, "cache is NULL"), (dict(src=None), EINVAL, "copy_src is NULL"), (dict(dst=None), EINVAL, "copy_dst is NULL"),
    (dict(count=-1), EINVAL, "count"), (dict(t=cache(P + 3 * M, P + 4 * M, P + 5 * M, page=32)), EINVAL, "differ"),
    (dict(t=cache(P + 3 * M, P + 4 * M, P + 5 * M, d=64)), EINVAL, "differ"), (dict(t=cache(P + 3 * M, P + 4 * M, P + 5 * M, Hkv=4)), EINVAL, "differ"),
    (dict(t=cache(P + 3 * M, P + 4 * M, P + 5 * M, dtype=pk.PK_BF16)), EINVAL, "differ"), (dict(t=cache(P + 3 * M, P + M, P + 5 * M)), EINVAL, "overlaps"),
    (dict(t=cache(P, P + 4 * M, P + 5 * M)), EINVAL, "overlap"), (dict(t=cache(blocks=9)), EINVAL, "overlap"), (dict(f=cache(page=8)), EUNSUPPORTED, "page_size"),
    (dict(f=cache(d=96)), EUNSUPPORTED, "{64, 128}"), (dict(dst=P + 2 * M), EINVAL, "overlaps"), (dict(src=P + 6 * M + 1), EINVAL, "aligned")])
def test_copies_refuse(change, code, word):
    a = dict(f=cache(), t=cache(), src=P + 6 * M, dst=P + 7 * M, count=4)
    a.update(change)
    refused(pk.lib().pk_kv_cache_copy(a["f"], a["t"], a["src"], a["dst"], a["count"], None), code, word)


def shared(**change):
    a = dict(cache=cache(), q=P + 3 * M, q_start=P + 4 * M, total=4, max_q=2, mask=P + 5 * M, table=P + 6 * M, most=8, lens=P + 7 * M, n=4, family=P + 8 * M, families=2,
             out=P + 9 * M, scale=0.1, Hq=32, out_dtype=pk.PK_BF16, ws=P + 10 * M, bytes=1 << 28)
    a.update(change)
    return pk.lib().pk_shared_tree_attn(a["cache"], a["q"], a["q_start"], a["total"], a["max_q"], a["mask"], a["table"], a["most"], a["lens"], a["n"], a["family"],
                                        a["families"], a["out"], a["scale"], a["Hq"], a["out_dtype"], a["ws"], a["bytes"], None)


@pytest.mark.parametrize("change, code, word", [
    (dict(cache=None), EINVAL, "cache is NULL"), (dict(cache=cache(d=96)), EUNSUPPORTED, "{64, 128}"), (dict(cache=cache(page=24)), EUNSUPPORTED, "page_size"),
    (dict(q=None), EINVAL, "NULL"), (dict(out=None), EINVAL, "NULL"), (dict(q_start=None), EINVAL, "NULL"), (dict(table=None), EINVAL, "NULL"), (dict(lens=None), EINVAL, "NULL"),
    (dict(family=None), EINVAL, "family_start is NULL"), (dict(families=-1), EINVAL, "families"), (dict(families=5), EINVAL, "families"), (dict(max_q=65), EUNSUPPORTED, "64"),
    (dict(max_q=-1), EINVAL, "max_q"), (dict(total=-1), EINVAL, "total_q"), (dict(total=1 << 31), EINVAL, "total_q"), (dict(Hq=12), EINVAL, "Hq"), (dict(Hq=0), EINVAL, "Hq"),
    (dict(scale=0.0), EINVAL, "scale"), (dict(scale=NAN), EINVAL, "scale"), (dict(out_dtype=pk.PK_F8), EINVAL, "out_dtype"), (dict(q=P + 8), EINVAL, "aligned"),
    (dict(out=P + 9 * M + 8), EINVAL, "aligned"), (dict(ws=None), EINVAL, "workspace"), (dict(ws=P + 64), EINVAL, "workspace"), (dict(bytes=4096), EINVAL, "smaller"),
    (dict(n=-1), EINVAL, "n <"), (dict(n=70000), EINVAL, "n <"), (dict(most=0), EINVAL, "max_blocks")])
def test_shared_attention_refuses(change, code, word):
    refused(shared(**change), code, word)


def verify(**change):
    a = dict(target=P, ts=1000, draft=P + M, ds=1000, dtype=pk.PK_BF16, vocab=1000, tokens=P + 2 * M, q_start=P + 3 * M, total=12, max_q=4, mask=P + 4 * M, n=3,
             temperature=P + 5 * M, accept=P + 6 * M, sample=P + 7 * M, keep=P + 8 * M, max_keep=4, count=P + 9 * M, after=P + 10 * M, ws=P + 11 * M, bytes=1 << 26)
    a.update(change)
    return pk.lib().pk_draft_verify(a["target"], a["ts"], a["draft"], a["ds"], a["dtype"], a["vocab"], a["tokens"], a["q_start"], a["total"], a["max_q"], a["mask"],
                                    a["n"], a["temperature"], a["accept"], a["sample"], a["keep"], a["max_keep"], a["count"], a["after"], a["ws"], a["bytes"], None)


@pytest.mark.parametrize("change, code, word", [
    (dict(target=None), EINVAL, "target is NULL"), (dict(tokens=None), EINVAL, "tokens is NULL"), (dict(q_start=None), EINVAL, "q_start is NULL"),
    (dict(accept=None), EINVAL, "accept_u is NULL"), (dict(sample=None), EINVAL, "sample_u is NULL"), (dict(keep=None), EINVAL, "keep is NULL"),
    (dict(count=None), EINVAL, "keep_count is NULL"), (dict(after=None), EINVAL, "next_token is NULL"), (dict(dtype=pk.PK_F8), EINVAL, "dtype"), (dict(vocab=0), EINVAL, "vocab"),
    (dict(vocab=(1 << 26) + 1, ts=1 << 27, ds=1 << 27), EUNSUPPORTED, "2^26"), (dict(ts=999), EINVAL, "target_stride"), (dict(ds=999), EINVAL, "draft_stride"),
    (dict(ts=-1000), EINVAL, "target_stride"), (dict(ts=1 << 60), EINVAL, "target_stride"), (dict(max_q=65), EUNSUPPORTED, "64"), (dict(max_q=-1), EINVAL, "max_q"),
    (dict(total=-1), EINVAL, "total_q"), (dict(n=-1), EINVAL, "n <"), (dict(n=65536), EINVAL, "n <"), (dict(max_keep=0), EINVAL, "max_keep"), (dict(target=P + 1), EINVAL, "aligned"),
    (dict(draft=P + M + 1), EINVAL, "aligned"), (dict(draft=P + M + 2, dtype=pk.PK_F32), EINVAL, "aligned"), (dict(mask=P + 4), EINVAL, "tree_mask"),
    (dict(temperature=P + 2), EINVAL, "temperature"), (dict(ws=None), EINVAL, "workspace"), (dict(bytes=100), EINVAL, "smaller"), (dict(keep=P + 2 * M), EINVAL, "overlaps"),
    (dict(after=P + 9 * M), EINVAL, "overlaps"), (dict(count=P + 5 * M), EINVAL, "overlaps"), (dict(after=P + 11 * M), EINVAL, "overlaps")])
def test_verify_refuses(change, code, word):
    refused(verify(**change), code, word)


def test_empty_calls_are_no_work():
    assert select(n=0, m=0, table=None, refs=None) == 0
    assert reserve(n=0, table=None, ws=None) == 0
    assert pk.lib().pk_kv_cache_copy(cache(), cache(), None, None, 0, None) == 0
    assert shared(n=0, families=0) == 0 and shared(total=0, q=None) == 0 and shared(max_q=0) == 0
    assert verify(n=0, target=None, ws=None) == 0


def test_sizes_of_workspaces():
    L = pk.lib()
    assert L.pk_kv_pages_workspace_bytes(0) == 0 and L.pk_kv_pages_workspace_bytes(1 << 31) == 0 and L.pk_kv_pages_workspace_bytes(1000) >= 12000
    assert L.pk_draft_verify_workspace_bytes(-1, 4, 100) == 0 and L.pk_draft_verify_workspace_bytes(1, 4, 0) == 0 and L.pk_draft_verify_workspace_bytes(4, 8, 32000) > 0
    assert L.pk_shared_tree_attn_workspace_bytes(4, 65, 8, 32, 8, 128) == 0 and L.pk_shared_tree_attn_workspace_bytes(4, 2, -1, 32, 8, 128) == 0
    assert L.pk_shared_tree_attn_workspace_bytes(4, 2, 8, 32, 8, 128) > 0 and L.pk_shared_tree_attn_workspace_bytes(4, 2, 8, 32, 8, 96) == 0
