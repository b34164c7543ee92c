"""Oracle of a feed-forward block and of the optimizer's step -- test infrastructure.

Plain numpy statements in fp64 of the textbook operations:

    AdamW   m = b1 m + (1 - b1) g,  v = b2 v + (1 - b2) g^2,
            p = p (1 - lr wd) - lr (m / (1 - b1^t)) / (sqrt(v / (1 - b2^t)) + eps)
            with g scaled by min(1, max_norm / (norm + 1e-6)) where a norm is given

8-bit states are e4m3 codes with a scale for each block of 256 elements, the block's
largest magnitude over 448; the second moment's codes are of its square root.
"""
from __future__ import annotations

import numpy as np

BLOCK = 256


def e4m3_values():
    """The value of each code (sign, four bits of exponent with bias 7, three of fraction; no
    infinities, 0x7F and 0xFF are NaN)."""
    c = np.arange(256)
    e, f = (c >> 3) & 15, c & 7
    x = np.where(e > 0, np.ldexp(1.0 + f / 8.0, e - 7), np.ldexp(f / 8.0, -6))
    x[(c & 127) == 127] = np.nan
    return np.where(c >= 128, -x, x)


def held(codes, scales):
    """What codes and their blocks' scales stand for."""
    codes = np.asarray(codes).reshape(-1)
    return e4m3_values()[codes] * np.repeat(np.asarray(scales, dtype=np.float64), BLOCK)[:len(codes)]


def block_scales(x):
    """The scale of each block of x."""
    x = np.abs(np.asarray(x, dtype=np.float64).reshape(-1))
    return np.array([x[i:i + BLOCK].max() / 448.0 for i in range(0, len(x), BLOCK)])


def adamw(p, g, m, v, t, lr, beta1, beta2, eps, weight_decay, norm=None, max_norm=np.inf):
    """(p, m, v) after a step, in fp64; v is the second moment itself."""
    p, g, m, v = (np.asarray(x, dtype=np.float64) for x in (p, g, m, v))
    if norm is not None:
        g = g * min(1.0, max_norm / (norm + 1e-6))
    m = beta1 * m + (1.0 - beta1) * g
    v = beta2 * v + (1.0 - beta2) * g * g
    change = (m / (1.0 - beta1 ** t)) / (np.sqrt(v / (1.0 - beta2 ** t)) + eps)
    return p - lr * weight_decay * p - lr * change, m, v
