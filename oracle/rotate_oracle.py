"""Float64 CPU oracle for norms and rotary positions of head rows.  TEST INFRASTRUCTURE ONLY, like cache_oracle."""
from __future__ import annotations

import numpy as np

__all__ = ["norm", "rotate"]


def norm(x, weight, eps):
    """x [..., 128]"""
    if weight is None:
        return x
    return x / np.sqrt((x * x).mean(-1, keepdims=True) + eps) * weight


def rotate(y, position, freqs, rotary, interleaved):
    """y [..., 128] at the positions [...], pair i by the angle position * freqs[i]."""
    out = y.copy()
    for i in range(rotary // 2):
        a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + rotary // 2)
        angle = np.asarray(position, np.float64) * freqs[i]
        c, s = np.cos(angle), np.sin(angle)
        out[..., a] = y[..., a] * c - y[..., b] * s
        out[..., b] = y[..., b] * c + y[..., a] * s
    return out
