"""Norms and position rotation of heads' rows in 64 bits (the definitions the kernels are
tested against)."""

import numpy as np


def frequencies(rotated, base):
    return base ** (-2.0 * np.arange(rotated // 2) / rotated)


def norm(x, w, eps):
    """Rows x [..., d] over the root of their mean square, times w [d]."""
    return x / np.sqrt((x * x).mean(-1, keepdims=True) + eps) * w


def rotate(x, positions, inv_freq, interleaved=False, scale=1.0):
    """Rows x [n, heads, d]: each pair of the first 2 * len(inv_freq) numbers (i and i + their
    number, or neighbours) turned by position * inv_freq[i] radians, times scale."""
    p = len(inv_freq)
    y = np.array(x, dtype=np.float64)
    t = (np.asarray(positions, np.float64)[:, None] * np.asarray(inv_freq, np.float64))[:, None, :]
    a, b = (slice(0, 2 * p, 2), slice(1, 2 * p, 2)) if interleaved else (slice(0, p), slice(p, 2 * p))
    y[..., a] = scale * (x[..., a] * np.cos(t) - x[..., b] * np.sin(t))
    y[..., b] = scale * (x[..., a] * np.sin(t) + x[..., b] * np.cos(t))
    return y
