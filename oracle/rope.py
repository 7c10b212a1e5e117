"""RMS norm of heads and rotation by position (test infrastructure only; plain numpy, float64, one formula per line).

    y_i = x_i * w_i / sqrt(mean of x_j^2 + eps)
    pair i: (y_i, y_{i + n}) of n pairs, or (y_2i, y_{2i+1}); turned by t = freq_i * position on axis_i
"""
import numpy as np


def qk_norm_rope(x, weight, eps, freq, axis, positions, adjacent):
    """x [rows, heads, D]; weight [D] or None; freq, axis [pairs]; positions [axes, rows].  Returns [rows, heads, D]."""
    y = np.array(x, dtype=np.float64)
    if weight is not None:
        y = y / np.sqrt((y ** 2).mean(axis=-1, keepdims=True) + float(np.float32(eps))) * np.asarray(weight, dtype=np.float64)
    out = y.copy()
    n = len(freq)
    for i in range(n):
        angle = np.asarray(positions[axis[i]], dtype=np.float64) * np.float64(np.float32(freq[i]))
        c, s = np.cos(angle)[:, None], np.sin(angle)[:, None]
        first, second = (2 * i, 2 * i + 1) if adjacent else (i, i + n)
        out[..., first] = y[..., first] * c - y[..., second] * s
        out[..., second] = y[..., second] * c + y[..., first] * s
    return out
