"""Plain statements in 64 bits of the operators on a language model's parameters.

TEST INFRASTRUCTURE ONLY: shares no code with the CUDA library and is never imported by it.

* orthogonalise: Y_0 = G / (|G|_F + eps), then `steps` times Y <- a Y + b (Y Y^T) Y + c (Y Y^T)^2 Y.
* step: v <- mu v + g; u = v or g + mu v; x <- (1 - lr weight_decay) x - lr scale orthogonalise(u).
* embed: out[t] = scale * table[ids[t]], a zero row where the id is negative or not below vocab.
* embed_grad: row v of worker m's gradient is scale * the sum of dout[m, t] over the t with ids[m, t] == v.
* layer_norm: (x - mean) / sqrt(variance + eps) * weight + bias per row; zero where the id is negative.
* layer_norm_grad: its derivative with respect to x, weight and bias, the latter two summed over each worker's rows.
* clip: norm per worker over all tensors; every entry times min(1, max_norm / (norm + eps)).
"""
from __future__ import annotations

import numpy as np


def singular_map(s, steps, coeffs):
    """What orthogonalise does to one (normalised) singular value."""
    a, b, c = coeffs
    for _ in range(steps):
        s = a * s + b * s ** 3 + c * s ** 5
    return s


def orthogonalise(g, steps, coeffs, eps):
    y = np.asarray(g, dtype=np.float64)
    y = y / (np.sqrt((y * y).sum(axis=(-2, -1), keepdims=True)) + eps)
    a, b, c = coeffs
    for _ in range(steps):
        p = y @ np.swapaxes(y, -1, -2)
        y = a * y + (b * p + c * (p @ p)) @ y
    return y


def step(x, v, g, mu, nesterov, lr, weight_decay, scale, steps, coeffs, eps):
    """(x, v) after the step; v None: without momentum."""
    x, g = np.asarray(x, dtype=np.float64), np.asarray(g, dtype=np.float64)
    u = g
    if v is not None:
        v = mu * np.asarray(v, dtype=np.float64) + g
        u = g + mu * v if nesterov else v
    return (1 - lr * weight_decay) * x - lr * scale * orthogonalise(u, steps, coeffs, eps), v


def embed(table, ids, scale):
    table = np.asarray(table, dtype=np.float64)
    out = np.zeros(ids.shape + table.shape[1:])
    there = (ids >= 0) & (ids < table.shape[0])
    out[there] = scale * table[ids[there]]
    return out


def embed_grad(dout, ids, vocab, scale):
    """[M, vocab, dim], and the same sum over magnitudes (what bounds the rounding of any order of summation)."""
    M, T = ids.shape
    total = np.zeros((M, vocab, dout.shape[-1]))
    size = np.zeros_like(total)
    for m in range(M):
        for t in range(T):
            if 0 <= ids[m, t] < vocab:
                total[m, ids[m, t]] += scale * dout[m, t].astype(np.float64)
                size[m, ids[m, t]] += abs(scale) * np.abs(dout[m, t].astype(np.float64))
    return total, size


def _centred(x, eps):
    x = np.asarray(x, dtype=np.float64)
    d = x - x.mean(-1, keepdims=True)
    rstd = 1 / np.sqrt((d * d).mean(-1, keepdims=True) + eps)
    return d * rstd, rstd


def layer_norm(x, weight, bias, eps, ids=None):
    """y, and xhat."""
    xhat, _ = _centred(x, eps)
    y = xhat * (1 if weight is None else np.asarray(weight, dtype=np.float64)) + (0 if bias is None else np.asarray(bias, dtype=np.float64))
    return (y, xhat) if ids is None else (np.where((ids >= 0)[..., None], y, 0.0), xhat)


def layer_norm_grad(dy, x, weight, eps, ids=None, dtotal=None):
    """(dx, dweight, dbias) for x [M, T, dim], and what bounds their rounding: the three sums' parts in magnitude."""
    there = np.ones(x.shape[:-1], dtype=bool) if ids is None else ids >= 0
    xhat, rstd = _centred(np.where(there[..., None], x, 0.0), eps)
    dy = np.where(there[..., None], np.asarray(dy, dtype=np.float64), 0.0)
    g = dy * (1 if weight is None else np.asarray(weight, dtype=np.float64))
    dx = rstd * (g - g.mean(-1, keepdims=True) - xhat * (g * xhat).mean(-1, keepdims=True))
    mg, mgx = np.abs(g).mean(-1, keepdims=True), np.abs(g * xhat).mean(-1, keepdims=True)
    size = rstd * (28 * np.abs(g) + 68 * mg + 40 * np.abs(xhat) * mg + (124 * np.abs(xhat) + 40) * mgx)
    if dtotal is not None:
        dx = dx + np.where(there[..., None], np.asarray(dtotal, dtype=np.float64), 0.0)
    sizes = size, (np.abs(dy) * (29 * np.abs(xhat) + 40)).sum(1), np.abs(dy * xhat).sum(1), np.abs(dy).sum(1)
    return dx, (dy * xhat).sum(1), dy.sum(1), sizes


def clip(grads, max_norm, eps):
    """(scaled tensors, norms) of tensors [M, ...]."""
    M = grads[0].shape[0]
    grads = [np.asarray(g, dtype=np.float64) for g in grads]
    norm = np.sqrt(sum((g.reshape(M, -1) ** 2).sum(1) for g in grads))
    c = np.minimum(1.0, max_norm / (norm + eps))
    return [g * c.reshape((M,) + (1,) * (g.ndim - 1)) for g in grads], norm
