"""Plain statements in 64 bits of the operators on a language model's parameters.

TEST INFRASTRUCTURE ONLY: shares no code with the CUDA library and is never imported by it.

* orthogonalise: Y_0 = G / (|G|_F + eps), then `steps` times Y <- a Y + b (Y Y^T) Y + c (Y Y^T)^2 Y.
* step: v <- mu v + g; u = v or g + mu v; x <- (1 - lr weight_decay) x - lr scale orthogonalise(u).
* embed: out[t] = scale * table[ids[t]], a zero row where the id is negative or not below vocab.
* embed_grad: row v of worker m's gradient is scale * the sum of dout[m, t] over the t with ids[m, t] == v.
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
