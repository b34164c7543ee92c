"""Oracle of a feed-forward block and of the optimizer's step -- test infrastructure.

Plain numpy statements in fp64 of the textbook operations:

    AdamW   m = b1 m + (1 - b1) g,  v = b2 v + (1 - b2) g^2,
            p = p (1 - lr wd) - lr (m / (1 - b1^t)) / (sqrt(v / (1 - b2^t)) + eps)
            with g scaled by min(1, max_norm / (norm + 1e-6)) where a norm is given

    gated   out = act(x Wg^T) (x Wu^T);  linear  out = act(x W^T + b) + residual;
            their gradients from the chain rule, with act SiLU, GELU (tanh) or none

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


def sigmoid_of(act, z):
    """(s, ds/dz) with act(z) = z sigmoid(s): SiLU, or GELU in its tanh form."""
    z = np.asarray(z, dtype=np.float64)
    if act == "silu":
        return z, np.ones_like(z)
    c = 2.0 * np.sqrt(2.0 / np.pi)
    return c * (z + 0.044715 * z ** 3), c * (1.0 + 3.0 * 0.044715 * z ** 2)


def activation(act, z):
    """(act(z), act'(z)) in fp64."""
    z = np.asarray(z, dtype=np.float64)
    if act == "none":
        return z, np.ones_like(z)
    s, ds = sigmoid_of(act, z)
    with np.errstate(over="ignore"):
        p = 1.0 / (1.0 + np.exp(-s))
        q = 1.0 / (1.0 + np.exp(s))  # 1 - p
    return z * p, p + z * p * q * ds


def gated_linear(x, w_gate, w_up, act):
    """(out, gate, up) in fp64."""
    x, wg, wu = (np.asarray(t, dtype=np.float64) for t in (x, w_gate, w_up))
    gate, up = x @ wg.T, x @ wu.T
    return activation(act, gate)[0] * up, gate, up


def gated_linear_grad(dout, x, w_gate, w_up, gate, up, act, add=0.0):
    """(dx, dw_gate, dw_up, dgate, dup) in fp64, from the saved gate and up."""
    dout, x, wg, wu, gate, up = (np.asarray(t, dtype=np.float64) for t in (dout, x, w_gate, w_up, gate, up))
    value, slope = activation(act, gate)
    dgate, dup = dout * up * slope, dout * value
    return dgate @ wg + dup @ wu + add, dgate.T @ x, dup.T @ x, dgate, dup


def linear(x, weight, bias, act, residual=0.0):
    """(out, z) in fp64; bias and residual may be 0."""
    z = np.asarray(x, dtype=np.float64) @ np.asarray(weight, dtype=np.float64).T + bias
    return activation(act, z)[0] + residual, z


def linear_grad(dout, x, weight, pre, act, add=0.0):
    """(dx, dweight, dbias, dz) in fp64, from the saved z (any with act "none")."""
    dout, x, w = (np.asarray(t, dtype=np.float64) for t in (dout, x, weight))
    dz = dout if act == "none" else dout * activation(act, pre)[1]
    return dz @ w + add, dz.T @ x, dz.sum(axis=0), dz
