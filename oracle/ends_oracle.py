"""fp64 oracle of what the two ends of a pipeline compute beside their layers, and of the norm over all gradients: embedding
and its gradient, token cross entropy and its gradient, global norm and clipping.  numpy, one formula a line; test
infrastructure only."""
from __future__ import annotations

import numpy as np


def embedding_fwd(ids, table, scale=1.0, positions=None, pos_table=None):
    """scale * table[id] + pos_table[position]; the term of an id outside its table is 0."""
    out = np.zeros((len(ids), table.shape[1]))
    for t, v in enumerate(ids):
        if 0 <= v < table.shape[0]:
            out[t] = scale * table[v]
        if pos_table is not None and 0 <= positions[t] < pos_table.shape[0]:
            out[t] += pos_table[positions[t]]
    return out


def embedding_bwd(ids, dy, vocab, scale=1.0):
    """(gradient [vocab, h], how often each id occurs, sums of absolute values)"""
    grad, mag, n = np.zeros((vocab, dy.shape[1])), np.zeros((vocab, dy.shape[1])), np.zeros(vocab, dtype=np.int64)
    for t, v in enumerate(ids):
        if 0 <= v < vocab:
            grad[v] += scale * dy[t]
            mag[v] += abs(scale) * np.abs(dy[t])
            n[v] += 1
    return grad, n, mag


def cross_entropy(x, targets, smoothing=0.0, g=1.0):
    """(losses, gradient of g * sum of the losses, probabilities)"""
    rows, vocab = x.shape
    ok = (targets >= 0) & (targets < vocab)
    with np.errstate(all="ignore"):
        m = x.max(axis=1, keepdims=True)
        e = np.exp(x - m)
        s = e.sum(axis=1, keepdims=True)
        log, m = np.log(s)[:, 0], m[:, 0]
        y = np.where(ok, targets, 0)
        at = np.arange(rows)
        loss = log + (m - x[at, y])   # the maximum and what is subtracted first: both may be the type's lowest value
        if smoothing:
            loss = (1 - smoothing) * loss + smoothing * (log + (m - x.mean(axis=1)))
        p = e / s
        dx = p - smoothing / vocab
        dx[at, y] -= 1 - smoothing
    return np.where(ok, loss, 0.0), np.where(ok[:, None], g * dx, 0.0), p


def grad_norm(tensors):
    """(sum of squares of the finite entries, number of the others)"""
    return (float(sum(np.square(t[np.isfinite(t)]).sum() for t in tensors)), int(sum((~np.isfinite(t)).sum() for t in tensors)))


def clip_factor(sum_sq, max_norm, eps):
    norm = float(np.sqrt(sum_sq)) + eps
    return min(1.0, max_norm / norm) if norm > 0 else 1.0
