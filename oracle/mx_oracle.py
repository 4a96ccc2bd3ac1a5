"""Float64 CPU oracle for numbers of 4 bits with a scale per 32 of them (OCP microscaling, MXFP4), as a cache holds them.

TEST INFRASTRUCTURE ONLY, like cache_oracle."""
from __future__ import annotations

import numpy as np

__all__ = ["NUMBERS", "encode", "decode"]

NUMBERS = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
LEAST, MOST, NAN = 2, 252, 255


def encode(x):
    """x [..., 128], numbers of bf16 in 64 bits -> codes [..., 128], scale bytes [..., 4].  The scale is the largest power of two 2^e with which
    the largest magnitude m 2^k does not need more than 6 1/2 steps of the format: e = k - 2 for m < 1.75, else k - 1; each number goes to the
    nearest one, of two as near to the one whose code is even."""
    x = np.asarray(x, np.float64)
    g = x.reshape(-1, 32)
    codes, scales = np.zeros(g.shape, np.int64), np.zeros(len(g), np.int64)
    finite = np.isfinite(g).all(1)
    top = np.abs(np.where(np.isfinite(g), g, 0.0)).max(1)
    m, k = np.frexp(top)                                   # top = m 2^k, m in [1/2, 1)
    e = np.where(top == 0, -10 ** 6, k - 1 - 2 + (m >= 0.875))
    e = np.clip(e, LEAST - 127, MOST - 127)
    size = np.abs(np.where(np.isfinite(g), g, 0.0)) / 2.0 ** e[:, None]
    far = np.abs(size[:, :, None] - NUMBERS)
    near = far == far.min(2, keepdims=True)
    order = np.where(np.arange(8) % 2 == 0, np.arange(8), np.arange(8) + 8)      # even codes first
    codes = np.where(near, order, 99).min(2) % 8 + 8 * np.signbit(g)
    codes = np.where(finite[:, None], codes, 0)
    scales = np.where(finite, e + 127, NAN)
    return codes.reshape(x.shape), scales.reshape(*x.shape[:-1], 4)


def decode(codes, scales):
    codes, scales = np.asarray(codes), np.asarray(scales)
    value = np.where(codes >= 8, -1.0, 1.0) * NUMBERS[codes % 8]
    size = np.where(scales == NAN, np.nan, 2.0 ** (scales.astype(np.float64) - 127))
    return value * np.repeat(size, 32, -1)
