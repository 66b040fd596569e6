"""ctypes binding of libpackinfer.so: argument marshalling only.

Function names mirror the C ABI (include/packinfer.h).  Tensors are torch
tensors on the GPU (device memory and streams come from PyTorch); lengths and
ids are host integer sequences.  There is no CPU fallback: if the library is
missing or a call fails, an exception is raised.
"""
from __future__ import annotations

import ctypes
import os
import struct
from typing import Optional, Sequence

import numpy as np

PK_BF16, PK_F32, PK_F8 = 0, 1, 2
PK_GROUP_ALIGN = 32
PK_KV_BLOCK = 32
PK_MAX_DRAFTS = 64

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libpackinfer.so")
_lib = None
_torch = None                           # the torch module, once lib() has loaded it
_dtype_codes = {}
_raw_stream = None                      # handle of a device's current stream, without a Stream object around it


class PackInferError(RuntimeError):
    pass


def lib():
    global _lib, _torch, _raw_stream
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise PackInferError(
            f"{LIB_PATH} is missing: build it with `python -m paper_2602_06072_amd.build`")
    # PyTorch owns the device memory and the streams: load its HIP runtime first so that the
    # library's libamdhip64 dependency resolves to the same, already initialised, runtime.
    import torch
    L = ctypes.CDLL(LIB_PATH)
    vp, i32, i64, f32, sz = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_float, ctypes.c_size_t
    ci = ctypes.c_int
    L.pk_pack_plan.restype = ci
    L.pk_pack_plan.argtypes = [vp, vp, vp, vp, i32, i64, i32, ctypes.POINTER(vp)]
    L.pk_plan_destroy.restype = None
    L.pk_plan_destroy.argtypes = [vp]
    for name in ("pk_plan_num_requests", "pk_plan_num_groups"):
        getattr(L, name).restype = i32
        getattr(L, name).argtypes = [vp]
    for name in ("pk_plan_buf_tokens", "pk_plan_unique_tokens", "pk_plan_serialized_words"):
        getattr(L, name).restype = i64
        getattr(L, name).argtypes = [vp]
    L.pk_plan_serialize.restype = i64
    L.pk_plan_serialize.argtypes = [vp, vp, i64]
    L.pk_kv_buf_bytes.restype = sz
    L.pk_kv_buf_bytes.argtypes = [vp, ci, ci, ci]
    L.pk_workspace_bytes.restype = sz
    L.pk_workspace_bytes.argtypes = [vp, ci, ci, ci, ci]
    L.pk_plan_bind.restype = ci
    L.pk_plan_bind.argtypes = [vp, ci, ci, ci, ci, vp, sz, vp]
    L.pk_kv_reorganize.restype = ci
    L.pk_kv_reorganize.argtypes = [vp, vp, vp, vp, i32, i32, i64, ci, ci, ci, vp, vp, sz, vp]
    for name in ("pk_packed_prefill_attn", "pk_padded_prefill_attn"):
        getattr(L, name).restype = ci
        getattr(L, name).argtypes = [vp, vp, vp, vp, vp, f32, ci, ci, ci, ci, ci, vp, sz, vp]
    L.pk_packed_decode_attn.restype = ci
    L.pk_packed_decode_attn.argtypes = [vp, vp, vp, vp, f32, ci, ci, ci, ci, ci, vp, sz, vp]
    L.pk_packed_mixed_step.restype = ci
    L.pk_packed_mixed_step.argtypes = [vp, vp, vp, vp, vp, vp, sz, vp, vp, vp, vp, vp, sz, f32, ci, ci, ci, ci, ci, vp]
    L.pk_packed_decode_attn_static.restype = ci
    L.pk_packed_decode_attn_static.argtypes = [vp, vp, vp, vp, f32, ci, ci, ci, ci, ci, vp]
    L.pk_padded_decode_attn.restype = ci
    L.pk_padded_decode_attn.argtypes = [vp, vp, vp, vp, vp, i32, i32, i64, vp, f32, ci, ci, ci, ci, ci, vp, sz, vp]
    L.pk_packed_decode_attn_grown.restype = ci
    L.pk_packed_decode_attn_grown.argtypes = [vp, vp, vp, vp, f32, i32, ci, ci, ci, ci, ci, vp, sz, vp]
    L.pk_kv_append.restype = ci
    L.pk_kv_append.argtypes = [vp, vp, vp, vp, i32, ci, ci, ci, vp, sz, vp]
    L.pk_regroup_due.restype = ci
    L.pk_regroup_due.argtypes = [vp, i32, ctypes.POINTER(i32), ctypes.POINTER(i64)]
    L.pk_pack_plan_tree.restype = ci
    L.pk_pack_plan_tree.argtypes = [vp, vp, i32, vp, vp, i32, vp, i64, i32, ctypes.POINTER(vp)]
    L.pk_trie_tree.restype = ci
    L.pk_trie_tree.argtypes = [vp, vp, i32, i32, vp, vp, ctypes.POINTER(i32), vp, ctypes.POINTER(i64)]
    L.pk_trie_partition.restype = ci
    L.pk_trie_partition.argtypes = [vp, vp, i32, i32, vp, vp, ctypes.POINTER(i64)]
    L.pk_plan_tune.restype = ci
    L.pk_plan_tune.argtypes = [vp, ci, i64]
    L.pk_plan_stat.restype = i64
    L.pk_plan_stat.argtypes = [vp, ci]
    for name, types in (("pk_qk_norm_rope", [vp] * 6 + [f32, vp, i64, ci, ci, ci, vp]),
                        ("pk_kv_cache_write", [vp, vp, vp, vp, i64, vp]),
                        ("pk_qkv_cache_write", [vp] * 8 + [f32, vp, i64, ci, vp]),
                        ("pk_kv_cache_read", [vp, vp, i32, vp, vp, i32, vp, vp, i64, vp]),
                        ("pk_tree_attn", [vp, vp, vp, i64, i32, vp, vp, i32, vp, i32, vp, f32, ci, ci, vp, sz, vp]),
                        ("pk_kv_cache_keep", [vp, vp, i32, vp, vp, i32, vp, i32, vp, vp, vp]),
                        ("pk_kv_pages_select", [vp, vp, vp, i32, i32, vp, i32, vp, vp, vp, vp, i64, i32, vp]),
                        ("pk_kv_pages_reserve", [vp, vp, vp, i32, i32, vp, vp, i64, i32, vp, vp, vp, vp, sz, vp]),
                        ("pk_kv_pages_compact", [vp, vp, i32, i32, vp, i64, vp, vp, vp, vp, i32, vp, sz, vp]),
                        ("pk_kv_cache_copy", [vp, vp, vp, vp, i32, vp]),
                        ("pk_shared_tree_attn", [vp, vp, vp, i64, i32, vp, vp, i32, vp, i32, vp, i32, vp, f32, ci, ci, vp, sz, vp]),
                        ("pk_draft_verify", [vp, i64, vp, i64, ci, i32, vp, vp, i64, i32, vp, i32, vp, vp, vp, vp, i32, vp, vp, vp, sz, vp])):
        getattr(L, name).restype = ci
        getattr(L, name).argtypes = types
    L.pk_tree_attn_workspace_bytes.restype = sz
    L.pk_tree_attn_workspace_bytes.argtypes = [i32, i32, ci, ci, ci]
    for name, types in (("pk_kv_pages_workspace_bytes", [i64]),
                        ("pk_shared_tree_attn_workspace_bytes", [i32, i32, i64, ci, ci, ci]),
                        ("pk_draft_verify_workspace_bytes", [i32, i64, i32])):
        getattr(L, name).restype = sz
        getattr(L, name).argtypes = types
    L.pk_last_error.restype = ctypes.c_char_p
    L.pk_last_error.argtypes = []
    _torch = torch
    _raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)
    _lib = L
    return L


EXPORTS = [
    "pk_pack_plan", "pk_plan_destroy", "pk_plan_num_requests", "pk_plan_num_groups",
    "pk_plan_buf_tokens", "pk_plan_unique_tokens", "pk_plan_serialized_words",
    "pk_plan_serialize", "pk_kv_buf_bytes", "pk_workspace_bytes", "pk_plan_bind",
    "pk_kv_reorganize", "pk_packed_prefill_attn", "pk_packed_decode_attn",
    "pk_padded_prefill_attn", "pk_padded_decode_attn", "pk_plan_stat", "pk_last_error",
    "pk_kv_append", "pk_packed_decode_attn_grown", "pk_regroup_due", "pk_trie_partition",
    "pk_pack_plan_tree", "pk_trie_tree", "pk_plan_tune", "pk_packed_decode_attn_static",
    "pk_packed_mixed_step", "pk_qk_norm_rope", "pk_kv_cache_write", "pk_qkv_cache_write",
    "pk_kv_cache_read", "pk_tree_attn", "pk_tree_attn_workspace_bytes", "pk_kv_cache_keep",
    "pk_kv_pages_select", "pk_kv_pages_reserve", "pk_kv_pages_compact", "pk_kv_pages_workspace_bytes", "pk_kv_cache_copy",
    "pk_shared_tree_attn", "pk_shared_tree_attn_workspace_bytes", "pk_draft_verify", "pk_draft_verify_workspace_bytes",
]
STATIC_SCRATCH_BYTES = 16 << 20
TUNE_DECODE_SPLIT = 0
TUNE_PREFILL_PIPELINE = 1
REGROUP_DRIFT, REGROUP_HEADROOM, REGROUP_DRIFT_WITHIN_BUDGET = 1, 2, 4


def _check(rc, what):
    if rc != 0:
        msg = lib().pk_last_error().decode()
        raise PackInferError(f"{what} failed ({rc}): {msg}")


def _i32(x) -> Optional[np.ndarray]:
    if x is None:
        return None
    return np.ascontiguousarray(np.asarray(x), dtype=np.int32)


def _ptr(a):
    try:
        return a.data_ptr()             # torch tensor
    except AttributeError:
        return None if a is None else a.ctypes.data


# The lengths of a batch as a bytes object: ctypes hands its buffer on as it is, where asking an array for its address (ndarray.ctypes) builds an object, 0.6 us each.
def _words(a):
    return None if a is None else a.tobytes()


def _dtype_code(t):
    if not _dtype_codes:
        import torch
        _dtype_codes.update({torch.bfloat16: PK_BF16, torch.float32: PK_F32})
    code = _dtype_codes.get(t.dtype)
    if code is None:
        raise PackInferError(f"unsupported dtype {t.dtype}")
    return code


# A call of a small batch is bound by what the host does per call, and half of that was here: torch.cuda.current_stream()
# alone, which resolves a device argument and builds a Stream object, takes 5 us of the 11 of a decode call.
def _stream(stream):
    if stream is not None:
        return stream.cuda_stream
    if _raw_stream is not None and _torch.cuda.is_initialized():
        return _raw_stream(_torch._C._cuda_getDevice())
    return _torch.cuda.current_stream().cuda_stream


class Plan:
    """Owner of a pk_plan*; created by pack_plan()."""

    def __init__(self, handle):
        self._h = ctypes.c_void_p(handle)
        self._ws = None                 # keeps the bound workspace alive

    def __del__(self):
        h, self._h = getattr(self, "_h", None), None
        if h and _lib is not None:
            _lib.pk_plan_destroy(h)

    @property
    def handle(self):
        return self._h

    num_requests = property(lambda s: lib().pk_plan_num_requests(s._h))
    num_groups = property(lambda s: lib().pk_plan_num_groups(s._h))
    buf_tokens = property(lambda s: lib().pk_plan_buf_tokens(s._h))
    unique_tokens = property(lambda s: lib().pk_plan_unique_tokens(s._h))

    def words(self) -> np.ndarray:
        n = lib().pk_plan_serialized_words(self._h)
        out = np.zeros(n, dtype=np.int32)
        got = lib().pk_plan_serialize(self._h, out.ctypes.data, n)
        if got != n:
            _check(int(got), "pk_plan_serialize")
        return out

    def groups(self):
        """Parsed view of the canonical words: a list of dicts(load, buf_tokens, buf_base, members, nodes).
        Plans of pack_plan: members = (req, prefix_off, L_P, suffix_off, L_Q), nodes = [].
        Plans of pack_plan_tree: nodes = (node id, off, len, parent index or -1),
        members = (req, node index or -1, suffix_off, suffix tokens)."""
        raw = self.words()
        w = raw.astype(np.int64) & 0xFFFFFFFF
        version, G = int(w[1]), int(w[3])
        pos, out = 10, []
        for _ in range(G):
            load = int(w[pos] | (w[pos + 1] << 32))
            bt = int(w[pos + 2] | (w[pos + 3] << 32))
            bb = int(w[pos + 4] | (w[pos + 5] << 32))
            pos += 6
            nodes = []
            if version == 2:
                nn, nm = int(w[pos]), int(w[pos + 1])
                pos += 2
                nodes = [tuple(int(x) for x in raw[pos + 4 * j: pos + 4 * j + 4]) for j in range(nn)]
                pos += 4 * nn
                mem = [tuple(int(x) for x in raw[pos + 4 * j: pos + 4 * j + 4]) for j in range(nm)]
                pos += 4 * nm
            else:
                nm = int(w[pos])
                pos += 1
                mem = [tuple(int(x) for x in raw[pos + 5 * j: pos + 5 * j + 5]) for j in range(nm)]
                pos += 5 * nm
            out.append(dict(load=load, buf_tokens=bt, buf_base=bb, members=mem, nodes=nodes))
        return out

    def stat(self, what: int) -> int:
        return int(lib().pk_plan_stat(self._h, what))

    def tune(self, knob: int, value: int) -> None:
        _check(lib().pk_plan_tune(self._h, int(knob), int(value)), "pk_plan_tune")
        self._ws = None

    def kv_buf_bytes(self, Hkv, d, dtype) -> int:
        return int(lib().pk_kv_buf_bytes(self._h, Hkv, d, dtype))

    def workspace_bytes(self, Hq, Hkv, d, dtype) -> int:
        return int(lib().pk_workspace_bytes(self._h, Hq, Hkv, d, dtype))


def pack_plan(kv_lens: Sequence[int], q_lens: Optional[Sequence[int]] = None,
              prefix_ids: Optional[Sequence[int]] = None,
              prefix_lens: Optional[Sequence[int]] = None,
              token_budget: int = 8192, headroom: int = 0) -> Plan:
    kv, ql, pid, pl = _i32(kv_lens), _i32(q_lens), _i32(prefix_ids), _i32(prefix_lens)
    for a in (ql, pid, pl):
        if a is not None and a.shape != kv.shape:
            raise PackInferError("pack_plan: array lengths differ")
    h = ctypes.c_void_p()
    rc = lib().pk_pack_plan(_words(kv), _words(ql), _words(pid), _words(pl), kv.shape[0],
                            int(token_budget), int(headroom), ctypes.byref(h))
    _check(rc, "pk_pack_plan")
    return Plan(h.value)


def pack_plan_tree(kv_lens: Sequence[int], q_lens: Optional[Sequence[int]],
                   node_parent: Sequence[int], node_len: Sequence[int], req_node: Sequence[int],
                   token_budget: int = 8192, headroom: int = 0) -> Plan:
    kv, ql, par, nl, rn = _i32(kv_lens), _i32(q_lens), _i32(node_parent), _i32(node_len), _i32(req_node)
    if (ql is not None and ql.shape != kv.shape) or rn.shape != kv.shape or par.shape != nl.shape:
        raise PackInferError("pack_plan_tree: array lengths differ")
    h = ctypes.c_void_p()
    rc = lib().pk_pack_plan_tree(_words(kv), _words(ql), kv.shape[0], _words(par), _words(nl), par.shape[0],
                                 _words(rn), int(token_budget), int(headroom), ctypes.byref(h))
    _check(rc, "pk_pack_plan_tree")
    return Plan(h.value)


def new_workspace(plan: Plan, Hq, Hkv, d, dtype, device="cuda"):
    nbytes = max(256, plan.workspace_bytes(Hq, Hkv, d, dtype))     # (a plan has loaded the library, and with it torch)
    return _torch.empty(nbytes, dtype=_torch.uint8, device=device)


def new_kv_buf(plan: Plan, Hkv, d, dtype, device="cuda", fill=None):
    import torch
    nbytes = max(256, plan.kv_buf_bytes(Hkv, d, dtype))
    buf = torch.empty(nbytes, dtype=torch.uint8, device=device)
    if fill is not None:
        buf.fill_(fill)
    return buf


def plan_bind(plan: Plan, Hq, Hkv, d, dtype, workspace, stream=None):
    rc = lib().pk_plan_bind(plan.handle, Hq, Hkv, d, dtype, _ptr(workspace),
                            workspace.nbytes, _stream(stream))
    _check(rc, "pk_plan_bind")
    plan._ws = workspace


def kv_reorganize(plan: Plan, k_pages, v_pages, block_table, kv_buf, workspace, stream=None):
    """k_pages, v_pages: [num_blocks, page, Hkv, d]; block_table: int32 [n, max_blocks] (device)."""
    nb, page, Hkv, d = k_pages.shape
    rc = lib().pk_kv_reorganize(
        plan.handle, _ptr(k_pages), _ptr(v_pages), _ptr(block_table), block_table.shape[1],
        page, nb, Hkv, d, _dtype_code(k_pages), _ptr(kv_buf), _ptr(workspace),
        workspace.nbytes, _stream(stream))
    _check(rc, "pk_kv_reorganize")
    plan._ws = workspace                # the call may have bound the plan to it


def _prefill(fn_name, plan, q, k, v, out, scale, workspace, stream):
    _, Hq, d = q.shape
    Hkv = k.shape[1]
    rc = getattr(lib(), fn_name)(
        plan.handle, _ptr(q), _ptr(k), _ptr(v), _ptr(out), float(scale), Hq, Hkv, d,
        _dtype_code(q), _dtype_code(out), _ptr(workspace),
        workspace.nbytes, _stream(stream))
    _check(rc, fn_name)
    plan._ws = workspace
    return out


def packed_prefill_attn(plan, q, k, v, out, scale, workspace, stream=None):
    return _prefill("pk_packed_prefill_attn", plan, q, k, v, out, scale, workspace, stream)


def padded_prefill_attn(plan, q, k, v, out, scale, workspace, stream=None):
    return _prefill("pk_padded_prefill_attn", plan, q, k, v, out, scale, workspace, stream)


def packed_decode_attn(plan, q, kv_buf, out, scale, Hkv, workspace, stream=None):
    n, Hq, d = q.shape
    rc = lib().pk_packed_decode_attn(
        plan.handle, _ptr(q), _ptr(kv_buf), _ptr(out), float(scale), Hq, Hkv, d,
        _dtype_code(q), _dtype_code(out), _ptr(workspace),
        workspace.nbytes, _stream(stream))
    _check(rc, "pk_packed_decode_attn")
    plan._ws = workspace
    return out


def packed_mixed_step(prefill_plan, q, k, v, out, prefill_workspace,
                      decode_plan, decode_q, kv_buf, decode_out, decode_workspace, scale, stream=None):
    """Prefill tiles and decode work items of one continuous-batching step in one launch."""
    _, Hq, d = q.shape
    Hkv = k.shape[1]
    rc = lib().pk_packed_mixed_step(
        prefill_plan.handle, _ptr(q), _ptr(k), _ptr(v), _ptr(out), _ptr(prefill_workspace),
        prefill_workspace.nbytes,
        decode_plan.handle, _ptr(decode_q), _ptr(kv_buf), _ptr(decode_out), _ptr(decode_workspace),
        decode_workspace.nbytes,
        float(scale), Hq, Hkv, d, _dtype_code(q), _dtype_code(out), _stream(stream))
    _check(rc, "pk_packed_mixed_step")
    prefill_plan._ws = prefill_workspace
    decode_plan._ws = decode_workspace
    return out, decode_out


def packed_decode_attn_static(plan, q, kv_buf, out, scale, Hkv, stream=None):
    """packed_decode_attn without a workspace: tables and partial results live in the library's
    fixed scratch array (for callers that cannot allocate device memory)."""
    n, Hq, d = q.shape
    rc = lib().pk_packed_decode_attn_static(
        plan.handle, _ptr(q), _ptr(kv_buf), _ptr(out), float(scale), Hq, Hkv, d,
        _dtype_code(q), _dtype_code(out), _stream(stream))
    _check(rc, "pk_packed_decode_attn_static")
    plan._ws = None
    return out


def packed_decode_attn_grown(plan, q, kv_buf, out, scale, grown, Hkv, workspace, stream=None):
    n, Hq, d = q.shape
    rc = lib().pk_packed_decode_attn_grown(
        plan.handle, _ptr(q), _ptr(kv_buf), _ptr(out), float(scale), int(grown), Hq, Hkv, d,
        _dtype_code(q), _dtype_code(out), _ptr(workspace),
        workspace.nbytes, _stream(stream))
    _check(rc, "pk_packed_decode_attn_grown")
    plan._ws = workspace
    return out


def kv_append(plan, k_new, v_new, kv_buf, step, workspace, stream=None):
    n, Hkv, d = k_new.shape
    rc = lib().pk_kv_append(
        plan.handle, _ptr(k_new), _ptr(v_new), _ptr(kv_buf), int(step), Hkv, d, _dtype_code(k_new),
        _ptr(workspace), workspace.nbytes, _stream(stream))
    _check(rc, "pk_kv_append")
    plan._ws = workspace
    return kv_buf


def trie_partition(seqs, min_prefix=1):
    """seqs: list of token-id sequences.  Returns (prefix_ids, prefix_lens, saved_tokens)."""
    n = len(seqs)
    lens = np.asarray([len(s) for s in seqs], dtype=np.int32)
    flat = np.ascontiguousarray(np.concatenate([np.asarray(s, dtype=np.int32) for s in seqs]) if n else
                                np.zeros(0, dtype=np.int32))
    ids = np.full(n, -1, dtype=np.int32)
    plens = np.zeros(n, dtype=np.int32)
    saved = ctypes.c_int64(0)
    rc = lib().pk_trie_partition(flat.ctypes.data, lens.ctypes.data, n, int(min_prefix),
                                 ids.ctypes.data, plens.ctypes.data, ctypes.byref(saved))
    _check(rc, "pk_trie_partition")
    return ids, plens, saved.value


def trie_tree(seqs, min_prefix=1):
    """seqs: list of token-id sequences.  Returns (node_parent, node_len, req_node, saved_tokens)."""
    n = len(seqs)
    lens = np.asarray([len(s) for s in seqs], dtype=np.int32)
    flat = np.ascontiguousarray(np.concatenate([np.asarray(s, dtype=np.int32) for s in seqs]) if n else
                                np.zeros(0, dtype=np.int32))
    par = np.zeros(max(n, 1), dtype=np.int32)
    nl = np.zeros(max(n, 1), dtype=np.int32)
    rn = np.full(n, -1, dtype=np.int32)
    nn, saved = ctypes.c_int32(0), ctypes.c_int64(0)
    rc = lib().pk_trie_tree(flat.ctypes.data, lens.ctypes.data, n, int(min_prefix), par.ctypes.data,
                            nl.ctypes.data, ctypes.byref(nn), rn.ctypes.data, ctypes.byref(saved))
    _check(rc, "pk_trie_tree")
    return par[:nn.value].copy(), nl[:nn.value].copy(), rn, saved.value


def regroup_due(plan, steps):
    """(flags, drift): flags is a bit set of REGROUP_DRIFT / REGROUP_HEADROOM / REGROUP_DRIFT_WITHIN_BUDGET."""
    flags, drift = ctypes.c_int32(0), ctypes.c_int64(0)
    rc = lib().pk_regroup_due(plan.handle, int(steps), ctypes.byref(flags), ctypes.byref(drift))
    _check(rc, "pk_regroup_due")
    return flags.value, drift.value


def padded_decode_attn(plan, q, k_pages, v_pages, block_table, out, scale, workspace, stream=None):
    n, Hq, d = q.shape
    nb, page, Hkv, _ = k_pages.shape
    rc = lib().pk_padded_decode_attn(
        plan.handle, _ptr(q), _ptr(k_pages), _ptr(v_pages), _ptr(block_table),
        block_table.shape[1], page, nb, _ptr(out), float(scale), Hq, Hkv, d,
        _dtype_code(q), _dtype_code(out), _ptr(workspace),
        workspace.nbytes, _stream(stream))
    _check(rc, "pk_padded_decode_attn")
    plan._ws = workspace
    return out


# --------------------------------------------------------------------------
# a decode step on a paged cache: norm, rotation, cache, drafted tokens
# --------------------------------------------------------------------------

_ROWS = struct.Struct("Pqqi4x")         # pk_rows; a bytes object is handed on as it is (a ctypes.Structure takes 1 us to fill)
_CACHE = struct.Struct("PPPqiiii")      # pk_cache
_ROPE = struct.Struct("PPqPiiii")       # pk_rope


def _need(ok, what):
    if not ok:
        raise PackInferError(what)


# (checks on the way of every call name what they refuse only where they refuse: a formatted message takes as long as the check)
def _rows(x, name, heads=None, d=None):
    """pk_rows of a tensor [tokens, heads, d] (any strides, columns contiguous); None: a null pointer.  A stride that leads
    nowhere, of one token or one head, may be anything in a tensor."""
    if x is None:
        return None
    shape = x.shape
    if len(shape) != 3 or (heads is not None and (shape[1] != heads or shape[2] != d)):
        raise PackInferError(f"{name} must be [tokens, heads, d]" + ("" if heads is None else f" with {heads} heads of {d} columns"))
    ts, hs, cs = x.stride()
    if cs != 1 and shape[2] != 1 and x.numel() != 0:
        raise PackInferError(f"{name} must have contiguous columns")
    code = _dtype_codes.get(x.dtype)
    return _ROWS.pack(x.data_ptr(), ts if shape[0] > 1 else 0, hs if shape[1] > 1 else 0, _dtype_code(x) if code is None else code)


def _vector(x, name, dtype, n=None):
    """Address of a contiguous tensor of the given type (and number of elements)."""
    if x is None:
        return None
    if x.dtype != dtype or not x.is_contiguous() or (n is not None and x.numel() != n):
        raise PackInferError(f"{name} must be contiguous, {dtype}" + ("" if n is None else f", {n} elements"))
    return x.data_ptr()


class KvCache:
    """Paged cache of keys and values (pk_cache).  k: [num_blocks, Hkv, page_size, d]; v: [num_blocks, Hkv, page_size / 4,
    d, 4], four tokens interleaved; with torch.float8_e4m3fn also scales: [num_blocks, Hkv, 2, page_size] of
    torch.float8_e8m0fnu, and with torch.bfloat16 none."""

    def __init__(self, k, v, scales=None):
        lib()
        f8 = k.dtype == _torch.float8_e4m3fn
        _need(f8 or k.dtype == _torch.bfloat16, "a cache is torch.float8_e4m3fn or torch.bfloat16")
        _need(k.dim() == 4, "k must be [num_blocks, Hkv, page_size, d]")
        self.num_blocks, self.Hkv, self.page_size, self.d = k.shape
        self.k, self.v, self.scales, self.dtype = k, v, scales, PK_F8 if f8 else PK_BF16
        _need(v.dtype == k.dtype and tuple(v.shape) == (self.num_blocks, self.Hkv, self.page_size // 4, self.d, 4),
              "v must be [num_blocks, Hkv, page_size / 4, d, 4] of k's type")
        _need((scales is not None) == f8, "scales belong to a cache in 8 bits, and to no other")
        _need(not f8 or (scales.dtype == _torch.float8_e8m0fnu and tuple(scales.shape) == (self.num_blocks, self.Hkv, 2, self.page_size)),
              "scales must be [num_blocks, Hkv, 2, page_size] of torch.float8_e8m0fnu")
        _need(all(x is None or x.is_contiguous() for x in (k, v, scales)), "the tensors of a cache must be contiguous")
        self.raw = _CACHE.pack(k.data_ptr(), v.data_ptr(), scales.data_ptr() if f8 else 0, self.num_blocks, self.page_size, self.Hkv, self.d, self.dtype)


def new_kv_cache(num_blocks, page_size, Hkv, d, dtype=PK_F8, device="cuda") -> KvCache:
    """A cache of zeros (with the scale that rows of zeros have)."""
    lib()
    t = _torch.float8_e4m3fn if dtype == PK_F8 else _torch.bfloat16
    zeros = lambda shape: _torch.zeros(shape, dtype=_torch.uint8 if t.itemsize == 1 else t, device=device).view(t)  # noqa: E731
    scales = _torch.ones((num_blocks, Hkv, 2, page_size), dtype=_torch.uint8, device=device).view(_torch.float8_e8m0fnu) if dtype == PK_F8 else None
    return KvCache(zeros((num_blocks, Hkv, page_size, d)), zeros((num_blocks, Hkv, page_size // 4, d, 4)), scales)


class Rope:
    """Rotary positions (pk_rope).  table: fp32 [max_pos, 2, rot_dim / 2], cosines and sines; positions: int32 [tokens] or
    [axes, tokens] (device); pair_axis: axis of every rotated pair (host, None: the first); interleaved: pairs are
    columns (2p, 2p + 1) instead of (p, p + rot_dim / 2)."""

    def __init__(self, table, positions, pair_axis=None, interleaved=False):
        lib()
        _need(table.dtype == _torch.float32 and table.dim() == 3 and table.shape[1] == 2 and table.is_contiguous(),
              "table must be contiguous fp32 [max_pos, 2, rot_dim / 2]")
        positions = positions if positions.dim() == 2 else positions[None]
        _need(positions.dtype == _torch.int32 and positions.dim() == 2 and (positions.stride(1) == 1 or positions.shape[1] <= 1),
              "positions must be int32 [axes, tokens]")
        pairs = table.shape[2]
        self.pair_axis = None if pair_axis is None else np.ascontiguousarray(pair_axis, dtype=np.uint8)
        _need(self.pair_axis is None or self.pair_axis.shape == (pairs,), "pair_axis must name an axis for each of the pairs")
        self.table, self.positions, self.tokens = table, positions, positions.shape[1]
        self.raw = _ROPE.pack(table.data_ptr(), positions.data_ptr(), positions.stride(0), 0 if pair_axis is None else self.pair_axis.ctypes.data,
                              table.shape[0], 2 * pairs, positions.shape[0], int(bool(interleaved)))


def _raw_rope(rope, tokens):
    if rope is None:
        return None
    _need(rope.tokens >= tokens, "the rotation has fewer positions than there are tokens")
    return rope.raw


def qk_norm_rope(q, k, q_out, k_out, q_weight=None, k_weight=None, eps=1e-6, rope: Optional[Rope] = None, stream=None):
    """Norm (where there is a weight) and rotation of q [tokens, Hq, d] and k [tokens, Hkv, d] into q_out and k_out."""
    L = lib()
    tokens, Hq, d = q.shape
    Hkv = k.shape[1]
    _need(k.shape[0] == tokens and q_out.shape == q.shape and k_out.shape == k.shape, "q, k, q_out, k_out: shapes differ")
    rc = L.pk_qk_norm_rope(_rows(q, "q"), _rows(k, "k", Hkv, d), _rows(q_out, "q_out"), _rows(k_out, "k_out"),
                           _vector(q_weight, "q_weight", q.dtype, d), _vector(k_weight, "k_weight", q.dtype, d), float(eps),
                           _raw_rope(rope, tokens), tokens, Hq, Hkv, d, _stream(stream))
    _check(rc, "pk_qk_norm_rope")
    return q_out, k_out


def kv_cache_write(cache: KvCache, k, v, slots, stream=None):
    """Rows of k and v [tokens, Hkv, d] into slots (int64 [tokens], -1: not written) of the cache."""
    L = lib()
    tokens = k.shape[0]
    _need(v.shape[0] == tokens, "k and v have different numbers of tokens")
    rc = L.pk_kv_cache_write(cache.raw, _rows(k, "k", cache.Hkv, cache.d), _rows(v, "v", cache.Hkv, cache.d),
                             _vector(slots, "slots", _torch.int64, tokens), tokens, _stream(stream))
    _check(rc, "pk_kv_cache_write")
    return cache


def qkv_cache_write(cache: KvCache, q, k, v, slots, q_out, q_weight=None, k_weight=None, eps=1e-6, rope: Optional[Rope] = None, stream=None):
    """qk_norm_rope and kv_cache_write in one launch: q into q_out, k (normed and rotated) and v into the cache."""
    L = lib()
    tokens, Hq, d = q.shape
    _need(k.shape[0] == tokens and v.shape[0] == tokens and q_out.shape == q.shape and d == cache.d, "q, k, v, q_out: shapes differ")
    rc = L.pk_qkv_cache_write(cache.raw, _rows(q, "q"), _rows(k, "k", cache.Hkv, d), _rows(v, "v", cache.Hkv, d),
                              _vector(slots, "slots", _torch.int64, tokens), _rows(q_out, "q_out"),
                              _vector(q_weight, "q_weight", q.dtype, d), _vector(k_weight, "k_weight", q.dtype, d), float(eps),
                              _raw_rope(rope, tokens), tokens, Hq, _stream(stream))
    _check(rc, "pk_qkv_cache_write")
    return q_out


def kv_cache_read(cache: KvCache, block_table, kv_lens, row_start, k_out, v_out, stream=None):
    """Tokens 0 .. kv_lens[i] - 1 of every request as rows row_start[i], ... of k_out and v_out [rows, Hkv, d]."""
    L = lib()
    n, max_blocks = block_table.shape
    _need(v_out.shape == k_out.shape, "k_out and v_out: shapes differ")
    rc = L.pk_kv_cache_read(cache.raw, _vector(block_table, "block_table", _torch.int32), max_blocks, _vector(kv_lens, "kv_lens", _torch.int32, n),
                            _vector(row_start, "row_start", _torch.int32, n), n, _rows(k_out, "k_out", cache.Hkv, cache.d),
                            _rows(v_out, "v_out", cache.Hkv, cache.d), k_out.shape[0], _stream(stream))
    _check(rc, "pk_kv_cache_read")
    return k_out, v_out


def new_tree_workspace(n, max_q, Hq, Hkv, d, device="cuda"):
    """Workspace of tree_attn for up to n requests of up to max_q drafted tokens; zeros, as its first use asks for."""
    nbytes = max(256, int(lib().pk_tree_attn_workspace_bytes(n, max_q, Hq, Hkv, d)))
    return _torch.zeros(nbytes, dtype=_torch.uint8, device=device)


def tree_attn(cache: KvCache, q, q_start, max_q, tree_mask, block_table, kv_lens, out, scale, workspace, stream=None):
    """Attention of the drafted tokens q [total, Hq, d] (request i: rows q_start[i] .. q_start[i + 1]) over the cache.
    tree_mask: int64 [total], bit j = drafted token j of the same request is seen (None: those before and itself)."""
    L = lib()
    total, Hq, d = q.shape
    n, max_blocks = block_table.shape
    _need(q.dtype == _torch.bfloat16 and q.is_contiguous() and out.is_contiguous() and out.shape == q.shape and d == cache.d,
          "q must be contiguous bf16 [total, Hq, d], out of the same shape")
    rc = L.pk_tree_attn(cache.raw, q.data_ptr(), _vector(q_start, "q_start", _torch.int32, n + 1), total, int(max_q),
                        _vector(tree_mask, "tree_mask", _torch.int64, total), _vector(block_table, "block_table", _torch.int32), max_blocks,
                        _vector(kv_lens, "kv_lens", _torch.int32, n), n, out.data_ptr(), float(scale), Hq, _dtype_code(out),
                        workspace.data_ptr(), workspace.nbytes, _stream(stream))
    _check(rc, "pk_tree_attn")
    return out


def kv_cache_keep(cache: KvCache, block_table, kv_lens, q_start, keep, keep_count, new_lens, *more, stream=None):
    """Drafted tokens keep[i, :keep_count[i]] (rising) of every request move up behind its context; new_lens receives
    the lengths with them.  The bound max_q of tree_attn may stand in front of keep."""
    L = lib()
    if not isinstance(keep, _torch.Tensor):
        _need(len(more) > 0, "kv_cache_keep takes [max_q], keep, keep_count and new_lens")
        max_q, keep, keep_count, new_lens, more = int(keep), keep_count, new_lens, more[0], more[1:]
        _need(0 <= max_q <= PK_MAX_DRAFTS, "need 0 <= max_q <= 64")
    _need(len(more) < 2 and not (more and stream is not None), "kv_cache_keep: one stream behind new_lens")
    stream = more[0] if more else stream
    n, max_blocks = block_table.shape
    _need(keep.dim() == 2 and keep.shape[0] == n, "keep must be [n, max_keep]")
    rc = L.pk_kv_cache_keep(cache.raw, _vector(block_table, "block_table", _torch.int32), max_blocks, _vector(kv_lens, "kv_lens", _torch.int32, n),
                            _vector(q_start, "q_start", _torch.int32, n + 1), n, _vector(keep, "keep", _torch.int32), keep.shape[1],
                            _vector(keep_count, "keep_count", _torch.int32, n), _vector(new_lens, "new_lens", _torch.int32, n), _stream(stream))
    _check(rc, "pk_kv_cache_keep")
    return new_lens


# --------------------------------------------------------------------------
# branching and judging: pages that requests share, and which drafted tokens stay
# --------------------------------------------------------------------------

def _batch(block_table, lens, pages, what=""):
    """(n, max_blocks, addresses of block table, lengths and pages) of a batch."""
    if block_table.dim() != 2:
        raise PackInferError(f"{what}block_table must be [n, max_blocks]")
    n, most = block_table.shape
    i32 = _torch.int32
    return n, most, _vector(block_table, what + "block_table", i32), _vector(lens, what + "lens", i32, n), _vector(pages, what + "pages", i32, n)


def kv_pages_select(block_table, lens, pages, rows_from, new_table, new_lens, new_pages, refs, page_size, stream=None):
    """Request i of the new batch is request rows_from[i] of the old one (outside of it: an empty one): forked, reordered and
    finished requests.  refs: int32 [num_blocks], how many requests hold a block."""
    L = lib()
    n, most, table, ls, ps = _batch(block_table, lens, pages)
    m, new_most, nt, nl, np_ = _batch(new_table, new_lens, new_pages, "new_")
    _need(new_most == most, "block_table and new_table differ in their max_blocks")
    rc = L.pk_kv_pages_select(table, ls, ps, n, most, _vector(rows_from, "rows_from", _torch.int32, m), m, nt, nl, np_,
                              _vector(refs, "refs", _torch.int32), refs.numel(), int(page_size), _stream(stream))
    _check(rc, "pk_kv_pages_select")
    return new_table, new_lens, new_pages


def new_pages_workspace(num_blocks, device="cuda"):
    """Workspace of kv_pages_reserve and kv_pages_compact; zeros, as its first use asks for."""
    nbytes = max(256, int(lib().pk_kv_pages_workspace_bytes(num_blocks)))
    return _torch.zeros(nbytes, dtype=_torch.uint8, device=device)


def kv_pages_reserve(block_table, lens, pages, grow, refs, page_size, served, copy_src, copy_dst, workspace, stream=None):
    """Pages for lens[i] + grow[i] tokens of every request, free blocks of the lowest numbers first; where a shared page with tokens of
    its own would be written, copy_src[i] -> copy_dst[i] (-1: none) is to be copied in every layer's cache (kv_cache_copy).
    served[i]: 1, or 0 where blocks ran out."""
    L = lib()
    n, most, table, ls, ps = _batch(block_table, lens, pages)
    i32 = _torch.int32
    rc = L.pk_kv_pages_reserve(table, ls, ps, n, most, _vector(grow, "grow", i32, n), _vector(refs, "refs", i32), refs.numel(), int(page_size),
                               _vector(served, "served", i32, n), _vector(copy_src, "copy_src", i32, n), _vector(copy_dst, "copy_dst", i32, n),
                               workspace.data_ptr(), workspace.nbytes, _stream(stream))
    _check(rc, "pk_kv_pages_reserve")
    return served


def kv_pages_compact(block_table, pages, refs, new_table, new_refs, copy_src, copy_dst, workspace, stream=None):
    """The blocks in use move to the lowest numbers: copy_src[k] -> copy_dst[k] (-1 behind the last one) are to be copied in every
    layer's cache; no more moves than these have room for.  new_table may be block_table."""
    L = lib()
    i32 = _torch.int32
    n, most, table, _, ps = _batch(block_table, pages, pages)
    _need(new_table.shape == block_table.shape and copy_src.numel() == copy_dst.numel(), "block_table and new_table, or copy_src and copy_dst: shapes differ")
    rc = L.pk_kv_pages_compact(table, ps, n, most, _vector(refs, "refs", i32), refs.numel(), _vector(new_table, "new_table", i32),
                               _vector(new_refs, "new_refs", i32, refs.numel()), _vector(copy_src, "copy_src", i32), _vector(copy_dst, "copy_dst", i32),
                               copy_src.numel(), workspace.data_ptr(), workspace.nbytes, _stream(stream))
    _check(rc, "pk_kv_pages_compact")
    return new_table


def kv_cache_copy(cache: KvCache, copy_src, copy_dst, to: Optional[KvCache] = None, stream=None):
    """Blocks copy_src[i] of the cache to blocks copy_dst[i], of `to` where it is given; numbers outside (-1) are passed over."""
    L = lib()
    to = cache if to is None else to
    rc = L.pk_kv_cache_copy(cache.raw, to.raw, _vector(copy_src, "copy_src", _torch.int32), _vector(copy_dst, "copy_dst", _torch.int32, copy_src.numel()),
                            copy_src.numel(), _stream(stream))
    _check(rc, "pk_kv_cache_copy")
    return to


def new_shared_tree_workspace(n, max_q, total_q, Hq, Hkv, d, device="cuda"):
    """Workspace of shared_tree_attn for up to n requests of up to max_q drafted tokens, total_q in all; zeros, as its first use
    asks for."""
    nbytes = max(256, int(lib().pk_shared_tree_attn_workspace_bytes(n, max_q, total_q, Hq, Hkv, d)))
    return _torch.zeros(nbytes, dtype=_torch.uint8, device=device)


def shared_tree_attn(cache: KvCache, q, q_start, max_q, tree_mask, block_table, kv_lens, family_start, out, scale, workspace, stream=None):
    """tree_attn for requests that have their leading pages in common: family g is requests family_start[g] ..
    family_start[g + 1] - 1 (int32 [families + 1]), whose shared pages are read once.  One number: no families, every request alone
    (faster where they are few or short)."""
    L = lib()
    total, Hq, d = q.shape
    n, max_blocks = block_table.shape
    _need(q.dtype == _torch.bfloat16 and q.is_contiguous() and out.is_contiguous() and out.shape == q.shape and d == cache.d,
          "q must be contiguous bf16 [total, Hq, d], out of the same shape")
    _need(family_start.numel() > 0, "family_start must be [families + 1]")
    rc = L.pk_shared_tree_attn(cache.raw, q.data_ptr(), _vector(q_start, "q_start", _torch.int32, n + 1), total, int(max_q),
                               _vector(tree_mask, "tree_mask", _torch.int64, total), _vector(block_table, "block_table", _torch.int32), max_blocks,
                               _vector(kv_lens, "kv_lens", _torch.int32, n), n, _vector(family_start, "family_start", _torch.int32),
                               family_start.numel() - 1, out.data_ptr(), float(scale), Hq, _dtype_code(out), workspace.data_ptr(), workspace.nbytes,
                               _stream(stream))
    _check(rc, "pk_shared_tree_attn")
    return out


def new_verify_workspace(n, total_q, vocab, device="cuda"):
    """Workspace of draft_verify for up to n requests with up to total_q tokens and vocab logits; zeros, as its first use asks for."""
    nbytes = max(256, int(lib().pk_draft_verify_workspace_bytes(n, total_q, vocab)))
    return _torch.zeros(nbytes, dtype=_torch.uint8, device=device)


def draft_verify(target, draft, tokens, q_start, max_q, tree_mask, temperature, accept_u, sample_u, keep, keep_count, next_token, workspace, stream=None):
    """Which drafted tokens of every request stay (keep [n, max_keep], keep_count [n], as kv_cache_keep takes them) and the token behind
    them (next_token [n]).  target, draft: logits [total, vocab] (bf16 or fp32, rows any distance apart; draft None: the tokens were not drawn);
    tokens int32 [total]; q_start, max_q, tree_mask as for tree_attn; temperature fp32 [n] (None: 1; 0: the largest logit); accept_u [total],
    sample_u [n]: fp32 random numbers from [0, 1)."""
    L = lib()
    i32, f32 = _torch.int32, _torch.float32
    total, vocab = target.shape
    n = q_start.numel() - 1
    _need(target.numel() == 0 or vocab == 1 or target.stride(1) == 1, "target must have contiguous rows")
    _need(draft is None or (draft.shape == target.shape and draft.dtype == target.dtype and (draft.numel() == 0 or vocab == 1 or draft.stride(1) == 1)),
          "draft must be of target's shape and type, with contiguous rows")
    _need(keep.dim() == 2 and keep.shape[0] == n, "keep must be [n, max_keep]")
    rc = L.pk_draft_verify(target.data_ptr(), target.stride(0) if total > 1 else vocab, None if draft is None else draft.data_ptr(),
                           vocab if draft is None or total < 2 else draft.stride(0), _dtype_code(target), vocab, _vector(tokens, "tokens", i32, total),
                           _vector(q_start, "q_start", i32), total, int(max_q), _vector(tree_mask, "tree_mask", _torch.int64, total), n,
                           _vector(temperature, "temperature", f32, n), _vector(accept_u, "accept_u", f32, total), _vector(sample_u, "sample_u", f32, n),
                           _vector(keep, "keep", i32), keep.shape[1], _vector(keep_count, "keep_count", i32, n),
                           _vector(next_token, "next_token", i32, n), workspace.data_ptr(), workspace.nbytes, _stream(stream))
    _check(rc, "pk_draft_verify")
    return keep, keep_count, next_token
