"""The oracle of the paged cache against hand-computed values, brute force and invariants."""
import math

import numpy as np
import pytest
import torch

from oracle import cache as oc


def test_values_of_the_format():
    v = oc.e4m3_values()
    assert v[0] == 0 and v[1] == 2.0 ** -9 and v[8] == 2.0 ** -6 and v[0x38] == 1.0 and v[0x7E] == 448.0 and v[0xFE] == -448.0
    assert math.isnan(v[0x7F]) and math.isnan(v[0xFF])
    want = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(v, want, equal_nan=True)


@pytest.mark.parametrize("top, E", [(448.0, 0), (448.5, 1), (1.0, -8), (1.75, -8), (1.7500001, -7), (2.0 ** -200, -126), (0.0, -126), (3.3e38, 120)])
def test_scale_is_the_smallest_that_holds_the_row(top, E):
    row = np.array([0.0, -top, top / 3])
    assert oc.scale_exponent(row) == E
    assert top <= math.ldexp(448.0, E)


def test_codes_are_the_nearest_values_and_ties_go_to_the_even_code():
    rng = np.random.default_rng(0)
    rows = np.concatenate([rng.normal(size=(50, 64)), rng.normal(size=(50, 64)) * np.exp(rng.normal(size=(50, 64)) * 3)])
    codes, E = oc.quantize(rows)
    grid = np.unique(oc.e4m3_values()[~np.isnan(oc.e4m3_values())])
    y = rows / 2.0 ** E[:, None]
    best = np.abs(y[..., None] - grid).min(-1)
    assert np.array_equal(np.abs(codes - y), best)
    tie, _ = oc.quantize(np.array([[448.0, 1.0625, 1.1875, 2.0 ** -10, 3 * 2.0 ** -10]]))       # halfway: 1 | 1.125 | 1.25; 0 | 2^-9 | 2^-8
    assert tie.tolist() == [[448.0, 1.0, 1.25, 0.0, 2.0 ** -8]]
    odd, e = oc.quantize(np.array([[math.inf, -math.inf, math.nan, 7.0]]))
    assert np.isnan(odd[0, :3]).all() and odd[0, 3] * 2.0 ** e[0] == 7.0


def test_rotation_by_hand_and_as_a_rotation():
    t = np.zeros((4, 2, 8))
    ang = np.arange(4)[:, None] * np.linspace(0.1, 1, 8)
    t[:, 0], t[:, 1] = np.cos(ang), np.sin(ang)
    x = np.random.default_rng(1).normal(size=(3, 2, 16))
    pos = np.array([[0, 3, 9], [2, 2, 2]])
    halves = oc.norm_rope(x, None, 0, t, pos, [0] * 4 + [1] * 4, False)
    z = (x[..., :8] + 1j * x[..., 8:]) * np.exp(1j * np.stack([ang[[0, 3, 3]][:, :4], ang[[2, 2, 2]][:, 4:]], 1).reshape(3, 1, 8))
    assert np.allclose(halves, np.concatenate([z.real, z.imag], -1))
    inter = oc.norm_rope(x, None, 0, t, pos, None, True)
    z = (x[..., 0::2] + 1j * x[..., 1::2]) * np.exp(1j * ang[[0, 3, 3]][:, None])
    assert np.allclose(inter[..., 0::2], z.real) and np.allclose(inter[..., 1::2], z.imag)
    n = oc.norm_rope(x, np.full(16, 2.0), 0.0, None, None, None, False)
    assert np.allclose((n * n).mean(-1), 4.0)


def test_tree_attention_against_a_masked_matrix_and_plain_causal_attention():
    rng = np.random.default_rng(2)
    T, L, Hq, Hkv, d = 5, 12, 4, 2, 8
    q, k, v = rng.normal(size=(T, Hq, d)), rng.normal(size=(L, Hkv, d)), rng.normal(size=(L, Hkv, d))
    mask = [0b1, 0b11, 0b101, 0b10011, 0b0]
    out, _ = oc.tree_attention(q, k, v, T, mask, 0.3)
    seen = torch.ones(T, L, dtype=torch.bool)
    for t in range(T):
        for j in range(T):
            seen[t, L - T + j] = bool(mask[t] >> j & 1)
    kk, vv = (torch.from_numpy(x).repeat_interleave(Hq // Hkv, 1).transpose(0, 1) for x in (k, v))
    for m, s in ((mask, seen), (None, torch.ones(T, L, dtype=torch.bool).tril(L - T))):
        want = torch.nn.functional.scaled_dot_product_attention(torch.from_numpy(q).transpose(0, 1)[None], kk[None], vv[None], s, scale=0.3)[0]
        assert np.allclose(oc.tree_attention(q, k, v, T, m, 0.3)[0], want.transpose(0, 1).numpy())
    alone, _ = oc.tree_attention(q, k[-T:], v[-T:], T, [0] * T, 0.3)
    assert not alone.any()
