"""Rotary positions, norms of query and key heads, and attention of packed sequences (fp64).

Definitions: rotary position embedding (Su et al. 2021), RMS norm (Zhang & Sennrich 2019), scaled
dot-product attention (Vaswani et al. 2017) with query heads that share key heads in groups
(Ainslie et al. 2023) and a causal mask aligned to the last key. Angles are taken in extended
precision: position times frequency, modulo a turn.
"""

import numpy as np

PAIRS, HALVES = 0, 1


def rotate(x, pos, freqs, axis_dims, pairing):
    """x [rows, heads, dim] turned to pos [rows, axes]; freqs: radians per position of every pair."""
    axis = np.repeat(np.arange(len(axis_dims)), [d // 2 for d in axis_dims])
    angle = pos.astype(np.longdouble)[:, axis] * np.asarray(freqs, np.longdouble)
    angle = np.fmod(angle, 2 * np.longdouble("3.14159265358979323846264338327950288")).astype(np.float64)
    cos, sin = np.cos(angle)[:, None], np.sin(angle)[:, None]
    half = len(axis)
    y = np.array(x, np.float64)
    first = slice(0, 2 * half, 2) if pairing == PAIRS else slice(0, half)
    second = slice(1, 2 * half, 2) if pairing == PAIRS else slice(half, 2 * half)
    a, b = np.array(y[..., first]), np.array(y[..., second])
    y[..., first], y[..., second] = a * cos - b * sin, a * sin + b * cos
    return y


def rms_norm(x, gain, eps):
    x = np.asarray(x, np.float64)
    return x / np.sqrt((x * x).mean(-1, keepdims=True) + eps) * gain


def attention(q, k, v, causal, scale):
    """One sequence: q [n, heads, dim], k, v [m, kv_heads, dim] -> (o, sum of p |v|), zeros where a row sees no key."""
    n, heads, dim = q.shape
    m, kv_heads, _ = k.shape
    group = heads // kv_heads
    o, a = np.zeros((n, heads, dim)), np.zeros((n, heads, dim))
    for h in range(heads):
        kh, vh = k[:, h // group], v[:, h // group]
        for i in range(n):
            seen = min(m, max(0, m - n + i + 1)) if causal else m
            if not seen:
                continue
            s = kh[:seen] @ q[i, h] * scale
            p = np.exp(s - s.max())
            p /= p.sum()
            o[i, h], a[i, h] = p @ vh[:seen], p @ np.abs(vh[:seen])
    return o, a
