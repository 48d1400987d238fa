"""Pins of the fp64 statements of the operators around the caches (oracle/operators_oracle.py)."""
import math

import numpy as np
import pytest
import torch

from oracle import operators_oracle as OP


def test_codes_of_hand_picked_blocks():
    row = np.zeros(64)
    # largest magnitude 4: scale 1, so every halfway point of the grid is hit exactly; ties go to the even code
    row[:14] = [4, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, -0.25, -0.75, 0.5, 1, 1.5, 2, 3]
    row[32] = 7.0        # stays with scale 1: the code of 6
    row[33] = -5.0       # halfway between 4 and 6: 4
    code, scale = OP.mx_round(row)
    assert scale.tolist() == [127, 127]
    assert code[:14].tolist() == [6, 0, 2, 2, 4, 4, 6, 8, 10, 1, 2, 3, 4, 5]
    assert code[32:34].tolist() == [7, 14]
    row[32] = 7.03125    # above 7: the next scale, 2 * 4 = 8
    code, scale = OP.mx_round(row)
    assert scale.tolist() == [127, 128] and code[32] == 6
    assert OP.mx_values(OP.mx_pack(code), scale)[[0, 32]].tolist() == [4.0, 8.0]


def test_codes_at_the_ends_of_the_range():
    top = np.zeros(32)
    top[0] = (2 - 2.0 ** -7) * 2.0 ** 127               # the largest bf16
    code, scale = OP.mx_round(top)
    assert scale[0] == 252 and code[0] == 7             # 6 * 2^125: finite in bf16
    tiny = np.zeros(32)
    tiny[0] = 2.0 ** -133                               # the smallest bf16
    code, scale = OP.mx_round(tiny)
    assert scale[0] == 2 and code[0] == 0
    assert OP.mx_round(np.zeros(32))[1][0] == 2
    for bad in (np.inf, -np.inf, np.nan):
        x = np.ones(64)
        x[3] = bad
        code, scale = OP.mx_round(x)
        assert scale.tolist() == [255, 125] and not code[:32].any()
        v = OP.mx_values(OP.mx_pack(code), scale)
        assert np.isnan(v[:32]).all() and np.array_equal(v[32:], np.ones(32))


def test_rounding_is_the_nearest_code_and_loses_what_is_stated():
    rng = np.random.default_rng(5)
    x = rng.standard_normal((4000, 64))
    x = torch.from_numpy(x).bfloat16().double().numpy()
    code, scale = OP.mx_round(x)
    v = OP.mx_values(OP.mx_pack(code), scale)
    rel = np.linalg.norm(v - x) / np.linalg.norm(x)
    assert 0.108 < rel < 0.116
    s = np.exp2(scale.astype(float) - 127).repeat(32, -1)
    d = np.abs(x - v) / s
    for g in OP.GRID:                                    # no other code is nearer
        assert (d <= np.minimum(np.abs(np.abs(x) / s - g), 99) + 1e-12).all()
    again = OP.mx_round(v)                               # what a cache holds is rounded to itself
    assert np.array_equal(OP.mx_values(OP.mx_pack(again[0]), again[1]), v)


def test_rotation_against_complex_numbers_and_its_invariants():
    rng = np.random.default_rng(6)
    x = rng.standard_normal((5, 3, 64))
    pos = rng.integers(0, 100000, (2, 5)).astype(np.int32)
    f = 10000.0 ** (-np.arange(16) / 16)
    axis = [i % 2 for i in range(16)]
    y, _ = OP.norm_rope(x, None, 0.0, pos, f, axis, True)
    z = (x[..., 0:32:2] + 1j * x[..., 1:32:2]) * np.exp(1j * pos[axis].T[:, None, :] * f)
    assert np.allclose(y[..., 0:32:2], z.real, atol=1e-11) and np.allclose(y[..., 1:32:2], z.imag, atol=1e-11)
    assert np.array_equal(y[..., 32:], x[..., 32:])
    # dot products of rotated rows depend on the distance of their positions alone
    a, _ = OP.norm_rope(x, None, 0.0, np.array([[3, 4, 5, 6, 7]]), f, [0] * 16, False)
    b, _ = OP.norm_rope(x, None, 0.0, np.array([[103, 104, 105, 106, 107]]), f, [0] * 16, False)
    assert np.allclose(np.einsum("thd,uhd->htu", a, a), np.einsum("thd,uhd->htu", b, b), atol=1e-10)
    n, _ = OP.norm_rope(x, np.ones(64), 0.0, pos, [], [], False)
    assert np.allclose((n * n).mean(-1), 1.0)


@pytest.mark.parametrize("t,n", [(5, 5), (3, 9), (1, 1), (6, 4)])
def test_prompt_attention_against_torch(t, n):
    rng = np.random.default_rng(7)
    q, k, v = rng.standard_normal((t, 16)), rng.standard_normal((n, 16)), rng.standard_normal((n, 16))
    out, lse, mass, _ = OP.prompt_attention(q, k, v)
    s = torch.from_numpy(q) @ torch.from_numpy(k).t() / math.sqrt(16)
    hidden = torch.arange(n)[None] > torch.arange(t)[:, None] + n - t
    s = s.masked_fill(hidden, -math.inf)
    seen = ~hidden.all(1)
    p = torch.softmax(s[seen], 1)
    assert np.allclose(out[seen.numpy()], (p @ torch.from_numpy(v)).numpy(), atol=1e-12)
    assert np.allclose(lse[seen.numpy()], (torch.logsumexp(s[seen], 1) / math.log(2)).numpy(), atol=1e-12)
    assert not out[~seen.numpy()].any() and np.isneginf(lse[~seen.numpy()]).all()
