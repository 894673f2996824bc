"""Norm of heads and rotation by position, in 64 bits, from the definition: each head x of a row becomes y = x / sqrt(mean(x^2) + eps) * w, and pairs of y's
first rotary_dim elements, as complex numbers, are multiplied by exp(i position freq)."""
from __future__ import annotations

import numpy as np


def norm_rotate(x, weight, eps, freq, rotary_dim, adjacent, positions):
    """x float64 [T][heads][D]; weight float64 [D] or None.  Returns the rows and, for each element, |a| + |b| of the pair it comes from
    (its own magnitude where it is not rotated): what the roundings of 32-bit arithmetic scale with."""
    y = np.array(x, np.float64)
    if weight is not None:
        y = y / np.sqrt((y * y).mean(-1, keepdims=True) + eps) * weight
    size = np.abs(y)
    n = rotary_dim // 2
    if n:
        i = np.arange(n)
        a, b = (2 * i, 2 * i + 1) if adjacent else (i, i + n)
        z = y[..., a] + 1j * y[..., b]
        z = z * np.exp(1j * (np.asarray(positions, np.float64)[:, None] * freq))[:, None, :]
        size[..., a] = size[..., b] = np.abs(y[..., a]) + np.abs(y[..., b])
        y[..., a], y[..., b] = z.real, z.imag
    return y, size
