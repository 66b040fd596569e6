"""Definitions of the paged cache in 8 bits, of norm and rotation, and of the attention of drafted tokens, in 64 bits.

Test infrastructure: shares no code with the library.  Arrays are numpy; a cache is token-major here (rows by slot
number), the layout of the library is taken apart by the tests from its description.
"""
import math

import numpy as np

E4M3_MAX = 448.0


def e4m3_values():
    """Value of every byte: sign, 4 exponent bits with bias 7, 3 fraction bits; no infinities, 0x7F and 0xFF are NaN."""
    out = np.empty(256)
    for b in range(256):
        e, f = (b >> 3) & 15, b & 7
        x = math.nan if (b & 127) == 127 else (f / 8 * 2.0 ** -6 if e == 0 else (1 + f / 8) * 2.0 ** (e - 7))
        out[b] = -x if b & 128 else x
    return out


def scale_exponent(row):
    """Smallest E >= -126 with the row's largest finite magnitude within 448 * 2^E."""
    finite = np.abs(row[np.isfinite(row)])
    top = float(finite.max()) if finite.size else 0.0
    E = -126
    if top > E4M3_MAX * 2.0 ** E:
        E = math.frexp(top)[1] - 10
        while top > math.ldexp(E4M3_MAX, E):
            E += 1
    return E


def quantize(rows):
    """rows [..., d] -> (values of the codes, exponents): nearest value of the format, ties to the even code."""
    rows = np.asarray(rows, dtype=np.float64)
    grid = np.unique(np.abs(e4m3_values()[:127]))                 # 0 .. 448, index = code
    flat = rows.reshape(-1, rows.shape[-1])
    codes, exps = np.empty_like(flat), np.empty(flat.shape[0], dtype=np.int64)
    for i, row in enumerate(flat):
        E = scale_exponent(row)
        exps[i] = E
        y = np.ldexp(np.where(np.isfinite(row), np.abs(row), 0.0), -E)
        hi = np.clip(np.searchsorted(grid, y), 1, len(grid) - 1)
        lo = hi - 1
        up = (y - grid[lo] > grid[hi] - y) | ((y - grid[lo] == grid[hi] - y) & (hi % 2 == 0))
        v = np.where(up, grid[hi], grid[lo]) * np.where(np.signbit(row), -1.0, 1.0)
        codes[i] = np.where(np.isfinite(row), v, np.nan)
    return codes.reshape(rows.shape), exps.reshape(rows.shape[:-1])


def norm_rope(x, weight, eps, table, positions, pair_axis, interleaved):
    """x [tokens, heads, d]; weight [d] or None; table [max_pos, 2, pairs] or None; positions [axes, tokens]."""
    x = np.asarray(x, dtype=np.float64)
    if weight is not None:
        x = x / np.sqrt((x * x).mean(-1, keepdims=True) + eps) * np.asarray(weight, dtype=np.float64)
    if table is None:
        return x
    table = np.asarray(table, dtype=np.float64)
    pairs = table.shape[2]
    y = x.copy()
    for p in range(pairs):
        pos = np.clip(positions[pair_axis[p] if pair_axis is not None else 0], 0, table.shape[0] - 1)
        c, s = table[pos, 0, p][:, None], table[pos, 1, p][:, None]
        i, j = (2 * p, 2 * p + 1) if interleaved else (p, p + pairs)
        y[..., i], y[..., j] = x[..., i] * c - x[..., j] * s, x[..., j] * c + x[..., i] * s
    return y


def tree_attention(q, k, v, drafts, mask, scale):
    """Attention of one request.  q [T, Hq, d] (T <= drafts: the drafted tokens' queries), k and v [len, Hkv, d], whose
    last `drafts` tokens are the drafted ones; mask: a word for each query, None: token t sees 0 .. t.
    Returns (out, sum of p |v|): what a row does not see is left out, a row that sees nothing is zero."""
    T, Hq, d = q.shape
    L, Hkv, _ = k.shape
    ctx = L - drafts
    out, spread = np.zeros((T, Hq, d)), np.zeros((T, Hq, d))
    for t in range(T):
        word = int(mask[t]) & (2 ** 64 - 1) if mask is not None else 2 ** (t + 1) - 1
        seen = [j for j in range(L) if j < ctx or (word >> (j - ctx)) & 1]
        if not seen:
            continue
        for h in range(Hq):
            g = h // (Hq // Hkv)
            s = scale * (k[seen, g] @ q[t, h])
            p = np.exp(s - s.max())
            p /= p.sum()
            out[t, h], spread[t, h] = p @ v[seen, g], p @ np.abs(v[seen, g])
    return out, spread
