"""CPU fp64 oracle of what stands around the decoder layers: embedding, loss over the vocabulary, gradient norm.

TEST INFRASTRUCTURE ONLY, like oracle/decoder_layer.py: the plain definitions in numpy fp64, sharing no code with the HIP path.
Pinned by tests/test_model_cpu.py (finite differences, closed forms, a library's cross entropy, planted mistakes).
"""
from __future__ import annotations

import numpy as np


def _inside(ids, V):
    return (ids >= 0) & (ids < V)


def embed_fwd(ids, table, scale=1.0):
    """x[t] = scale * table[ids[t]]; an id outside [0, V) gives a row of zeros."""
    x = np.zeros((len(ids), table.shape[1]))
    for t, v in enumerate(ids):
        if 0 <= v < table.shape[0]:
            x[t] = scale * table[v]
    return x


def embed_bwd(ids, dx, V, scale=1.0, G=None):
    """scale * the sum of the rows of dx by id, added to G where it is given."""
    out = np.zeros((V, dx.shape[1])) if G is None else np.array(G, dtype=np.float64)
    ok = _inside(ids, V)
    np.add.at(out, ids[ok], scale * dx[ok])
    return out


def loss_fwd(logits, labels, eps=0.0, z=0.0):
    """(rows, lse, counted): row = lse - (1-eps) l_y - eps mean_v l_v + z lse^2; rows whose label is outside [0, V) give 0.
    A row with nothing but -inf: lse -inf, loss +inf."""
    T, V = logits.shape
    rows, lse, counted = np.zeros(T), np.zeros(T), _inside(labels, V)
    for t in np.flatnonzero(counted):
        l = logits[t]
        top = np.max(l)
        if np.isneginf(top):
            rows[t], lse[t] = np.inf, -np.inf
            continue
        with np.errstate(invalid="ignore"):
            lse[t] = top + np.log(np.sum(np.exp(l - top)))
        r = lse[t] - (1.0 - eps) * l[labels[t]]
        if eps:
            r -= eps * np.mean(l)
        if z:
            r += z * lse[t] ** 2
        rows[t] = r
    return rows, lse, counted


def loss_total(rows, counted, mean=True):
    n = int(np.sum(counted))
    if n == 0:
        return 0.0, 0
    return float(np.sum(rows)) / (n if mean else 1), n


def loss_bwd(logits, labels, lse, up, eps=0.0, z=0.0, V_pad=None):
    """up[t] * d row / d logits, zeros in the columns V .. V_pad-1, in rows that are not counted and in rows with lse = -inf."""
    T, V = logits.shape
    d = np.zeros((T, V if V_pad is None else V_pad))
    for t in np.flatnonzero(_inside(labels, V)):
        if np.isneginf(lse[t]):
            continue
        with np.errstate(invalid="ignore"):
            g = np.exp(logits[t] - lse[t]) * (1.0 + 2.0 * z * lse[t]) - eps / V
        g[labels[t]] -= 1.0 - eps
        d[t, :V] = up[t] * g
    return d


def clip(grads, max_norm, grad_scale=1.0):
    """(norm, coef, nonfinite) of the gradients grad_scale * g."""
    norm = abs(grad_scale) * np.sqrt(sum(float(np.sum(np.square(g))) for g in grads))
    if not np.isfinite(norm):
        return norm, 0.0, 1
    return norm, (max_norm / norm if norm > max_norm else 1.0), 0
