"""Helpers of the tests of the feed-forward block: inputs, calls in canary-filled buffers, and
checks against the oracle in fp64.

Tolerances (U = 2^-24, half a step of fp32). A tensor-core product adds 16 terms a step to an
fp32 sum; a step may drop what lies below 2^-22 of the magnitudes added so far, so a product of
length K is off by at most (K / 16 + 4) 2^-22 of its sum of magnitudes; K splits join with up to
64 roundings more (64 U). The activation z sigmoid(s): 2^(-s log2 e) has an argument off by 8 U |s|
(gelu's s has three roundings of its own) and two approximations of 2^-22 each, so with T = 2^-20 +
8 U min(|s|, 90) the sigmoid is off by T of itself, the value by T |value|, and the slope
p (1 + z (1 - p) ds) by p (1 + |z ds|) (T + 4 U). No activation's slope exceeds 1.13. Below 2^-126 the
sigmoid is 0. Rounded operands and results are off by half a step of bf16, 2^-8."""
from __future__ import annotations

import numpy as np
import torch

import oracle
from train_util import HALF, U32, Guarded, dev, host, within

BF, F32 = torch.bfloat16, torch.float32
STEP = 2.0 ** -22
ACTS = {"none": 0, "silu": 1, "gelu": 2}
TINY = 1e-37


def rand(*shape, seed=0, std=1.0, dtype=BF):
    g = torch.Generator(device="cpu").manual_seed(seed)
    return (torch.randn(*shape, generator=g) * std).to(dtype).to(dev())


def length(K):
    return (K / 16 + 4) * STEP + 64 * U32


def sigmoid_error(act, z):
    """(s, ds, T)"""
    s, ds = oracle.sigmoid_of(act, z)
    return s, ds, 2.0 ** -20 + 8 * U32 * np.minimum(np.abs(s), 90.0)


def value_error(act, z, dz):
    """How far act(z) may be off for z off by dz."""
    if act == "none":
        return dz
    v, _ = oracle.activation(act, z)
    return 1.13 * dz + sigmoid_error(act, z)[2] * (np.abs(v) + 1.13 * dz) + TINY


def slope_error(act, z):
    if act == "none":
        return np.zeros_like(z)
    s, ds, T = sigmoid_error(act, z)
    with np.errstate(over="ignore"):
        p = 1.0 / (1.0 + np.exp(-s))
    return p * (1.0 + np.abs(z * ds)) * (T + 4 * U32) + TINY


def rounded(x, err):
    """The bound of a bf16 result."""
    return err + HALF[BF] * (np.abs(x) + err) + TINY


def check_gated(x, wg, wu, act, out, gate=None, up=None, where=""):
    X, G, W = host(x).reshape(-1, x.shape[-1]), host(wg), host(wu)
    o, g, u = oracle.gated_linear(X, G, W, act)
    eg, eu = (length(X.shape[1]) * (np.abs(X) @ np.abs(w).T) for w in (G, W))
    a = oracle.activation(act, g)[0]
    ea = value_error(act, g, eg)
    flat = lambda t: host(t).reshape(-1, t.shape[-1])  # noqa: E731
    within(flat(out), o, rounded(o, np.abs(a) * eu + np.abs(u) * ea + ea * eu + 2 * U32 * np.abs(o)), where + " out")
    if gate is not None:
        within(flat(gate), g, rounded(g, eg), where + " gate")
        within(flat(up), u, rounded(u, eu), where + " up")


def check_gated_grad(dout, x, wg, wu, gate, up, act, add, dx, dwg, dwu, where=""):
    flat = lambda t: host(t).reshape(-1, t.shape[-1])  # noqa: E731
    D, X, G, W, g, u = flat(dout), flat(x), host(wg), host(wu), flat(gate), flat(up)
    A = 0.0 if add is None else flat(add)
    rx, rg, ru, dg, du = oracle.gated_linear_grad(D, X, G, W, g, u, act, A)
    eg = np.abs(D * u) * slope_error(act, g) + 4 * U32 * np.abs(dg)
    eu = np.abs(D) * value_error(act, g, 0.0 * g) + 2 * U32 * np.abs(du)
    eg, eu = (e + HALF[BF] * (np.abs(z) + e) + TINY for e, z in ((eg, dg), (eu, du)))
    mg, mu = np.abs(dg) + eg, np.abs(du) + eu
    if dx is not None:
        e = eg @ np.abs(G) + eu @ np.abs(W) + length(2 * G.shape[0]) * (mg @ np.abs(G) + mu @ np.abs(W)) + 2 * U32 * np.abs(A)
        within(flat(dx), rx, rounded(rx, e), where + " dx")
    for got, want, e, m, n in ((dwg, rg, eg, mg, "dw_gate"), (dwu, ru, eu, mu, "dw_up")):
        if got is not None:
            within(host(got), want, rounded(want, e.T @ np.abs(X) + length(X.shape[0]) * (m.T @ np.abs(X))), f"{where} {n}")


def check_linear(x, w, bias, act, residual, out, pre=None, where=""):
    flat = lambda t: host(t).reshape(-1, t.shape[-1])  # noqa: E731
    X, W = flat(x), host(w)
    b = 0.0 if bias is None else host(bias)
    r = 0.0 if residual is None else flat(residual) if isinstance(residual, torch.Tensor) else residual
    o, z = oracle.linear(X, W, b, act, r)
    e = length(X.shape[1]) * (np.abs(X) @ np.abs(W).T) + U32 * (np.abs(z) + np.abs(b))
    within(flat(out), o, rounded(o, value_error(act, z, e) + 2 * U32 * (np.abs(o) + np.abs(r))), where + " out")
    if pre is not None:
        within(flat(pre), z, rounded(z, e), where + " pre")


def check_linear_grad(dout, x, w, pre, act, add, dx, dw, db, where=""):
    flat = lambda t: host(t).reshape(-1, t.shape[-1])  # noqa: E731
    D, X, W = flat(dout), flat(x), host(w)
    Z = D if pre is None else flat(pre)
    A = 0.0 if add is None else flat(add) if isinstance(add, torch.Tensor) else add
    rx, rw, rb, dz = oracle.linear_grad(D, X, W, Z, act, A)
    e32 = 0.0 * dz if act == "none" else np.abs(D) * slope_error(act, Z) + 2 * U32 * np.abs(dz)
    e = 0.0 * dz if act == "none" else e32 + HALF[BF] * (np.abs(dz) + e32) + TINY
    m = np.abs(dz) + e
    if dx is not None:
        within(flat(dx), rx, rounded(rx, e @ np.abs(W) + length(W.shape[0]) * (m @ np.abs(W)) + 2 * U32 * np.abs(A)), where + " dx")
    if dw is not None:
        within(host(dw), rw, rounded(rw, e.T @ np.abs(X) + length(X.shape[0]) * (m.T @ np.abs(X))), where + " dweight")
    if db is not None:
        # a thread adds up to N / 8 rows one after another, then 8 warps and up to 608 runs
        err = e32.sum(0) + (len(D) / 8 + 620) * U32 * (np.abs(dz) + e32).sum(0)
        within(host(db), rb, err + HALF[db.dtype] * (np.abs(rb) + err) + TINY, where + " dbias")


def workspace(size, *sizes, gd=None):
    n = size(*sizes)
    if gd is not None:
        return gd.empty(max(1, n), dtype=torch.uint8)
    return torch.full((max(1, n),), 0xFF, dtype=torch.uint8, device=dev())


__all__ = ["ACTS", "BF", "F32", "Guarded", "check_gated", "check_gated_grad", "check_linear", "check_linear_grad", "dev", "host", "rand",
           "workspace"]
