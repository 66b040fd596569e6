"""What the calls of the paged cache refuse: wrong arguments give a code and a message before anything is launched
(no GPU involved), and empty calls are no work."""
import ctypes

import numpy as np
import pytest

from paper_2602_06072_amd import binding as pk

EINVAL, EUNSUPPORTED = -1, -3
P = 1 << 20                                 # an address that is never read


def rows(data=P, ts=1024, hs=128, dtype=pk.PK_BF16):
    return pk._ROWS.pack(data, ts, hs, dtype)


def cache(k=P, v=P, scales=P, blocks=10, page=16, Hkv=8, d=128, dtype=pk.PK_F8):
    return pk._CACHE.pack(k, v, scales, blocks, page, Hkv, d, dtype)


def rope(table=P, positions=P, stride=4, axis=None, max_pos=100, rot=128, axes=1, interleaved=0):
    return pk._ROPE.pack(table, positions, stride, 0 if axis is None else axis.ctypes.data, max_pos, rot, axes, interleaved)


def refused(rc, code, word):
    assert rc == code, pk.lib().pk_last_error()
    assert word in pk.lib().pk_last_error().decode(), pk.lib().pk_last_error()


BAD_AXES = np.array([0] * 63 + [3], np.uint8)
F32, NAN = pk.PK_F32, float("nan")


@pytest.mark.parametrize("change, code, word", [
    (dict(q=None), EINVAL, "q is NULL"), (dict(k=None), EINVAL, "k is NULL"), (dict(q_out=None), EINVAL, "q_out"), (dict(k_out=None), EINVAL, "k_out"),
    (dict(q=rows(0)), EINVAL, "q is NULL"), (dict(q=rows(P + 2)), EINVAL, "16 bytes"), (dict(k=rows(ts=1020)), EINVAL, "16 bytes"),
    (dict(k=rows(hs=-128)), EINVAL, "stride"), (dict(k=rows(dtype=F32)), EINVAL, "another dtype"), (dict(k_out=rows(dtype=F32)), EINVAL, "another dtype"),
    (dict(q=rows(dtype=pk.PK_F8)), EINVAL, "dtype"), (dict(q_out=rows(hs=64)), EINVAL, "apart"), (dict(q_out=rows(ts=512, hs=128)), EINVAL, "apart"),
    (dict(tokens=-1), EINVAL, "tokens"), (dict(tokens=1 << 31), EINVAL, "tokens"), (dict(Hq=0), EINVAL, "Hq"), (dict(Hkv=-1), EINVAL, "Hkv"),
    (dict(d=100), EUNSUPPORTED, "multiple of 8"), (dict(d=264), EUNSUPPORTED, "256"), (dict(eps=-1.0), EINVAL, "eps"), (dict(eps=NAN), EINVAL, "eps"),
    (dict(wq=P + 4), EINVAL, "weights"), (dict(rope=rope(table=0)), EINVAL, "table"), (dict(rope=rope(table=P + 8)), EINVAL, "table"), (dict(rope=rope(positions=0)), EINVAL, "positions"),
    (dict(rope=rope(rot=136)), EINVAL, "rot_dim"), (dict(rope=rope(rot=24)), EUNSUPPORTED, "rot_dim"), (dict(rope=rope(max_pos=0)), EINVAL, "max_pos"),
    (dict(rope=rope(axes=0)), EINVAL, "n_axes"), (dict(rope=rope(interleaved=2)), EINVAL, "interleaved"), (dict(rope=rope(axes=3, axis=BAD_AXES)), EINVAL, "pair_axis")])
def test_norm_and_rotation_refuse(change, code, word):
    a = dict(q=rows(ts=4096), k=rows(), q_out=rows(ts=4096), k_out=rows(), wq=P, wk=P, eps=1e-6, rope=rope(), tokens=4, Hq=32, Hkv=8, d=128)
    a.update(change)
    refused(pk.lib().pk_qk_norm_rope(a["q"], a["k"], a["q_out"], a["k_out"], a["wq"], a["wk"], a["eps"], a["rope"], a["tokens"], a["Hq"], a["Hkv"], a["d"], None), code, word)


CACHES = [(dict(cache=None), EINVAL, "cache is NULL"), (dict(cache=cache(k=0)), EINVAL, "NULL"), (dict(cache=cache(scales=0)), EINVAL, "NULL"),
          (dict(cache=cache(v=P + 8)), EINVAL, "aligned"), (dict(cache=cache(page=8)), EUNSUPPORTED, "page_size"), (dict(cache=cache(page=0)), EUNSUPPORTED, "page_size"),
          (dict(cache=cache(d=96)), EUNSUPPORTED, "{64, 128}"), (dict(cache=cache(dtype=F32)), EINVAL, "cache dtype"), (dict(cache=cache(blocks=0)), EINVAL, "num_blocks"),
          (dict(cache=cache(Hkv=0)), EINVAL, "Hkv")]


@pytest.mark.parametrize("change, code, word", CACHES + [
    (dict(k=None), EINVAL, "k is NULL"), (dict(v=None), EINVAL, "v is NULL"), (dict(v=rows(dtype=F32)), EINVAL, "another dtype"), (dict(slots=None), EINVAL, "slots"),
    (dict(tokens=-2), EINVAL, "tokens"), (dict(k=rows(P + 1)), EINVAL, "16 bytes")])
def test_cache_write_refuses(change, code, word):
    a = dict(cache=cache(), k=rows(), v=rows(), slots=P, tokens=4)
    a.update(change)
    refused(pk.lib().pk_kv_cache_write(a["cache"], a["k"], a["v"], a["slots"], a["tokens"], None), code, word)
    if "k" not in change:
        refused(pk.lib().pk_qkv_cache_write(a["cache"], rows(ts=4096), a["k"], a["v"], a["slots"], rows(ts=4096), None, None, 0.0, None, a["tokens"], 32, None), code, word)


TABLES = [(dict(table=None), EINVAL, "block_table"), (dict(lens=None), EINVAL, "kv_lens"), (dict(max_blocks=0), EINVAL, "max_blocks"), (dict(max_blocks=1 << 30), EINVAL, "max_blocks"),
          (dict(n=-1), EINVAL, "n < 65536"), (dict(n=70000), EINVAL, "n < 65536")]


@pytest.mark.parametrize("change, code, word", CACHES + TABLES + [
    (dict(start=None), EINVAL, "row_start"), (dict(k_out=None), EINVAL, "k_out"), (dict(v_out=rows(dtype=F32)), EINVAL, "another dtype"), (dict(v_out=rows(hs=64)), EINVAL, "apart"), (dict(rows=-1), EINVAL, "rows")])
def test_cache_read_refuses(change, code, word):
    a = dict(cache=cache(), table=P, max_blocks=4, lens=P, start=P, n=3, k_out=rows(), v_out=rows(), rows=50)
    a.update(change)
    refused(pk.lib().pk_kv_cache_read(a["cache"], a["table"], a["max_blocks"], a["lens"], a["start"], a["n"], a["k_out"], a["v_out"], a["rows"], None), code, word)


@pytest.mark.parametrize("change, code, word", CACHES + TABLES + [
    (dict(q=None), EINVAL, "q, out"), (dict(out=P + 8), EINVAL, "aligned"), (dict(q_start=None), EINVAL, "q_start"), (dict(Hq=12), EINVAL, "Hq"), (dict(max_q=65), EUNSUPPORTED, "64"),
    (dict(max_q=-1), EINVAL, "max_q"), (dict(total=-1), EINVAL, "total_q"), (dict(scale=0.0), EINVAL, "scale"), (dict(scale=float("inf")), EINVAL, "scale"), (dict(out_dtype=pk.PK_F8), EINVAL, "out_dtype"),
    (dict(ws=None), EINVAL, "workspace"), (dict(ws=P + 128), EINVAL, "workspace"), (dict(ws_bytes=16), EINVAL, "workspace smaller")])
def test_attention_refuses(change, code, word):
    a = dict(cache=cache(), q=P, q_start=P, total=20, max_q=10, mask=P, table=P, max_blocks=4, lens=P, n=3, out=P, scale=0.1, Hq=32, out_dtype=pk.PK_BF16, ws=P, ws_bytes=1 << 40)
    a.update(change)
    refused(pk.lib().pk_tree_attn(a["cache"], a["q"], a["q_start"], a["total"], a["max_q"], a["mask"], a["table"], a["max_blocks"], a["lens"], a["n"], a["out"], a["scale"], a["Hq"],
                                  a["out_dtype"], a["ws"], a["ws_bytes"], None), code, word)


@pytest.mark.parametrize("change, code, word", CACHES + TABLES + [
    (dict(q_start=None), EINVAL, "q_start"), (dict(keep=None), EINVAL, "keep"), (dict(count=None), EINVAL, "keep"), (dict(new=None), EINVAL, "new_lens"), (dict(new=P), EINVAL, "kv_lens itself"), (dict(max_keep=-1), EINVAL, "max_keep")])
def test_keep_refuses(change, code, word):
    a = dict(cache=cache(), table=P, max_blocks=4, lens=P, q_start=P, n=3, keep=P, max_keep=5, count=P, new=2 * P)
    a.update(change)
    refused(pk.lib().pk_kv_cache_keep(a["cache"], a["table"], a["max_blocks"], a["lens"], a["q_start"], a["n"], a["keep"], a["max_keep"], a["count"], a["new"], None), code, word)


def test_empty_calls_are_no_work():
    L = pk.lib()
    r, c = rows(ts=4096), cache()
    assert L.pk_qk_norm_rope(r, rows(), r, rows(), None, None, 0.0, None, 0, 32, 8, 128, None) == 0
    assert L.pk_kv_cache_write(c, rows(0), rows(0), None, 0, None) == 0
    assert L.pk_qkv_cache_write(c, r, rows(), rows(), None, r, None, None, 0.0, None, 0, 32, None) == 0
    assert L.pk_kv_cache_read(c, None, 4, None, None, 0, rows(), rows(), 50, None) == 0
    assert L.pk_kv_cache_read(c, P, 4, P, P, 2, rows(0), rows(0), 0, None) == 0
    for total, max_q, n in ((0, 5, 3), (5, 0, 3), (5, 5, 0)):
        assert L.pk_tree_attn(c, None, None, total, max_q, None, P, 4, P, n, None, 0.1, 32, 0, None, 0, None) == 0
    assert L.pk_kv_cache_keep(c, None, 4, None, None, 0, None, 0, None, None, None) == 0


def test_the_binding_refuses_tensors_that_do_not_fit():
    import torch
    bf16, f8 = torch.bfloat16, torch.float8_e4m3fn
    c = pk.new_kv_cache(4, 16, 2, 64, device="cpu")
    x = torch.zeros(3, 2, 64, dtype=bf16)
    slots = torch.zeros(3, dtype=torch.int64)
    e = pk.PackInferError
    for bad in (lambda: pk.KvCache(c.k, c.v), lambda: pk.KvCache(c.k, c.k, c.scales), lambda: pk.KvCache(c.k.transpose(1, 2), c.v, c.scales),
                lambda: pk.KvCache(c.k.view(torch.uint8), c.v, c.scales), lambda: pk.kv_cache_write(c, x[:, :1], x, slots), lambda: pk.kv_cache_write(c, x, x, slots[:2]),
                lambda: pk.kv_cache_write(c, x, x, slots.int()), lambda: pk.kv_cache_write(c, x.half(), x.half(), slots), lambda: pk.kv_cache_write(c, x[..., ::2], x, slots),
                lambda: pk.Rope(torch.zeros(4, 2, 32).double(), slots.int()), lambda: pk.Rope(torch.zeros(4, 2, 32), slots), lambda: pk.Rope(torch.zeros(4, 2, 32), slots.int(), [0] * 31),
                lambda: pk.qk_norm_rope(x, x, x[:2], x), lambda: pk.qk_norm_rope(x, x, x, x, torch.zeros(63, dtype=bf16)), lambda: pk.qk_norm_rope(x, x, x, x, torch.zeros(64)),
                lambda: pk.qk_norm_rope(x, x, x, x, rope=pk.Rope(torch.zeros(4, 2, 32), slots[:2].int()))):
        with pytest.raises(e):
            bad()


def test_the_structures_are_those_of_the_header():
    assert (pk._ROWS.size, pk._CACHE.size, pk._ROPE.size) == (32, 48, 48)
    assert ctypes.sizeof(ctypes.c_void_p) == 8
