"""Plain fp64 statements of the operators around the caches: norm and rotation of query and key rows, causal
attention over prompts of different lengths, rounding of rows to 4 bits and their values.

TEST INFRASTRUCTURE ONLY: numpy, no product code.
"""
from __future__ import annotations

import numpy as np

GRID = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def norm_rope(x, weight, eps, pos, inv_freq, axis, interleaved):
    """x [tokens, H, D] fp64, pos [axes, tokens]: rows normed (weight None: not) and rotated.  Also returns the magnitude of the
    pair that every element comes from, which bounds what rounding of the products can do."""
    y = x.copy()
    if weight is not None:
        y = y * weight / np.sqrt((y * y).mean(-1, keepdims=True) + eps)
    out, size = y.copy(), np.abs(y)
    half = len(inv_freq)
    for i in range(half):
        a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + half)
        t = pos[axis[i]].astype(np.float64) * inv_freq[i]
        c, s = np.cos(t)[:, None], np.sin(t)[:, None]
        out[..., a] = y[..., a] * c - y[..., b] * s
        out[..., b] = y[..., a] * s + y[..., b] * c
        size[..., a] = size[..., b] = np.abs(y[..., a]) + np.abs(y[..., b])
    return out, size


def prompt_attention(q, k, v):
    """One head of one sequence: q [t, D] are the last of the tokens that k, v [n, D] hold.  Returns (out, lse in log2 units, sum of
    weight times |v|, largest sum of |q_d k_d| / sqrt(D) over the visible keys); a query that sees nothing: zeros, -inf."""
    t, D = q.shape
    n = k.shape[0]
    out, mass = np.zeros((t, D)), np.zeros((t, D))
    lse, big = np.full(t, -np.inf), np.zeros(t)
    for i in range(t):
        m = n - t + i + 1
        if m <= 0:
            continue
        s = k[:m] @ q[i] / np.sqrt(D)
        top = s.max()
        e = np.exp(s - top)
        p = e / e.sum()
        out[i], mass[i] = p @ v[:m], p @ np.abs(v[:m])
        lse[i] = (top + np.log(e.sum())) * np.log2(np.e)
        big[i] = (np.abs(k[:m]) @ np.abs(q[i])).max() / np.sqrt(D)
    return out, lse, mass, big


def mx_round(x):
    """Rows x [..., D] fp64 (bf16 values): codes 0 .. 15 [..., D] and scale bytes [..., D / 32]."""
    b = np.asarray(x, dtype=np.float64).reshape(x.shape[:-1] + (x.shape[-1] // 32, 32))
    fine = np.isfinite(b).all(-1)
    top = np.where(fine, np.abs(np.where(np.isfinite(b), b, 0.0)).max(-1), 1.0)
    m, e = np.frexp(top)                       # top = m 2^e, 0.5 <= m < 1
    e = np.where(top > 0, e - 3 + (m > 0.875), -125)
    e = np.clip(e, -125, 125)
    y = np.abs(np.where(fine[..., None], b, 0.0)) * np.exp2(-e.astype(np.float64))[..., None]
    # nearest code, ties to the even one: distances to all eight
    d = np.abs(y[..., None] - GRID)
    best = d.min(-1, keepdims=True)
    near = d == best
    code = np.where(near, np.arange(8), 99)
    low = code.min(-1)
    high = np.where(near, np.arange(8), -1).max(-1)
    code = np.where(low % 2 == 0, low, high)
    code = code + 8 * np.signbit(b)
    code = np.where(fine[..., None], code, 0)
    scale = np.where(fine, e + 127, 255)
    return code.reshape(x.shape).astype(np.uint8), scale.astype(np.uint8)


def mx_pack(code):
    return (code[..., 0::2] | (code[..., 1::2] << 4)).astype(np.uint8)


def mx_values(packed, scale):
    """fp64 values of packed codes [..., D / 2] with scale bytes [..., D / 32]."""
    code = np.stack([packed & 15, packed >> 4], -1).reshape(packed.shape[:-1] + (2 * packed.shape[-1],))
    v = GRID[code & 7] * np.where(code & 8, -1.0, 1.0)
    s = np.where(scale == 255, np.nan, np.exp2(scale.astype(np.float64) - 127))
    return (v.reshape(s.shape + (32,)) * s[..., None]).reshape(v.shape)
