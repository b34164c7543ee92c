"""Oracle of training and scoring the refiner's last layer -- test infrastructure.

Plain numpy statements in fp64 of the norm in front of the output projection,
the cross entropy of given tokens under the projection, their gradients, and
the clipping of a set of gradients by their common norm. The paper trains
nothing; the operations are the textbook ones:

    layer norm       out = (x - mean) rstd w + b over the last dimension
    cross entropy    loss[r] = lse[r] - logits[r, t_r]; rows whose target is
                     outside [0, V) are not scored and have no gradient
    clipping         g * min(1, max_norm / (norm + 1e-6)), norm over all tensors

The gradients are written from the chain rule, independently of the library's
arrangement of them; the pins compare them with torch's autograd in fp64 and
with differences.
"""
from __future__ import annotations

import numpy as np

from .lmhead import lm_head_logits


def layer_norm(x, weight, bias=None, eps=1e-5):
    """(out [N, d], mean [N], rstd [N]) in fp64."""
    x = np.asarray(x, dtype=np.float64)
    mean = x.mean(axis=1)
    rstd = 1.0 / np.sqrt(((x - mean[:, None]) ** 2).mean(axis=1) + eps)
    out = (x - mean[:, None]) * rstd[:, None] * np.asarray(weight, dtype=np.float64)
    return out + (0.0 if bias is None else np.asarray(bias, dtype=np.float64)), mean, rstd


def layer_norm_grad(dout, x, weight, mean, rstd):
    """(dx, dweight, dbias) in fp64, from the saved mean and rstd."""
    dout, x = np.asarray(dout, dtype=np.float64), np.asarray(x, dtype=np.float64)
    mean, rstd = (np.asarray(v, dtype=np.float64)[:, None] for v in (mean, rstd))
    xhat = (x - mean) * rstd
    dxhat = dout * np.asarray(weight, dtype=np.float64)
    # out depends on x directly, through the mean and through rstd
    d_direct = dxhat * rstd
    d_mean = -d_direct.sum(axis=1, keepdims=True)
    d_rstd = (dxhat * (x - mean)).sum(axis=1, keepdims=True)
    d_var = d_rstd * -0.5 * rstd ** 3
    dx = d_direct + d_mean / x.shape[1] + d_var * 2.0 * (x - mean) / x.shape[1]
    return dx, (dout * xhat).sum(axis=0), dout.sum(axis=0)


def scored_rows(targets, V):
    """Rows that have a target."""
    t = np.asarray(targets)
    return np.nonzero((t >= 0) & (t < V))[0]


def lm_head_loss(hidden, weight, targets):
    """(loss [N], lse [N]) in fp64; 0 for rows that are not scored."""
    N, V = len(targets), len(weight)
    loss, lse = np.zeros(N), np.zeros(N)
    rows = scored_rows(targets, V)
    if len(rows):
        x = lm_head_logits(np.asarray(hidden)[rows], weight)
        m = x.max(axis=1)
        lse[rows] = m + np.log(np.exp(x - m[:, None]).sum(axis=1))
        loss[rows] = lse[rows] - x[np.arange(len(rows)), np.asarray(targets)[rows]]
    return loss, lse


def lm_head_loss_grad(hidden, weight, targets, lse, dloss):
    """(d_hidden [N, d], d_weight [V, d]) in fp64, and the gradient of the logits of
    the scored rows (for error bounds)."""
    h, w = np.asarray(hidden, dtype=np.float64), np.asarray(weight, dtype=np.float64)
    V = w.shape[0]
    rows = scored_rows(targets, V)
    d_hidden, d_weight = np.zeros_like(h), np.zeros_like(w)
    if not len(rows):
        return d_hidden, d_weight, np.zeros((0, V))
    g = np.exp(lm_head_logits(h[rows], w) - np.asarray(lse, dtype=np.float64)[rows, None])
    g[np.arange(len(rows)), np.asarray(targets)[rows]] -= 1.0
    g *= np.asarray(dloss, dtype=np.float64)[rows, None]
    d_hidden[rows] = g @ w
    d_weight[:] = g.T @ h[rows]
    return d_hidden, d_weight, g


def clip_grad_norm(grads, max_norm):
    """(scaled gradients, norm) in fp64."""
    grads = [np.asarray(g, dtype=np.float64) for g in grads]
    norm = np.sqrt(sum(float((g * g).sum()) for g in grads))
    scale = max_norm / (norm + 1e-6)
    if scale >= 1.0:
        scale = 1.0
    return [g * scale for g in grads], norm
