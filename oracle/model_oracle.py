"""fp64 CPU oracle of a model's two ends and the update of its matrices (test infrastructure only): token
rows and their gradient, the cross entropy of a vocabulary with its gradients, Newton-Schulz updates.

Written from the definitions in numpy float64.  Shares nothing with the HIP path.
"""
from __future__ import annotations

import numpy as np


def counts(ids, vocab):
    ids = np.asarray(ids, dtype=np.int64)
    return (ids >= 0) & (ids < vocab)


def embed(table, ids, scale):
    table = np.asarray(table, dtype=np.float64)
    on = counts(ids, len(table))
    out = np.zeros((len(ids), table.shape[1]))
    out[on] = scale * table[np.asarray(ids, dtype=np.int64)[on]]
    return out


def embed_backward(ids, dout, vocab, scale):
    """(the dense gradient, the sum of the absolute values of its terms, terms of each row)"""
    on = counts(ids, vocab)
    at, rows = np.asarray(ids, dtype=np.int64)[on], scale * np.asarray(dout, dtype=np.float64)[on]
    grad, size = np.zeros((vocab, dout.shape[1])), np.zeros((vocab, dout.shape[1]))
    np.add.at(grad, at, rows)
    np.add.at(size, at, np.abs(rows))
    return grad, size, np.bincount(at, minlength=vocab)


def logits(x, w, scale):
    return scale * (np.asarray(x, dtype=np.float64) @ np.asarray(w, dtype=np.float64).T)


def head_loss(x, w, targets, scale):
    """(loss, lse)"""
    z = logits(x, w, scale)
    top = z.max(axis=1, keepdims=True)
    lse = top[:, 0] + np.log(np.exp(z - top).sum(axis=1))
    on = counts(targets, z.shape[1])
    loss = np.zeros(len(z))
    at = np.nonzero(on)[0]
    loss[at] = lse[at] - z[at, np.asarray(targets, dtype=np.int64)[at]]
    return loss, lse


def head_slope(x, w, targets, dloss, scale):
    """The gradient of the scaled products <x, w>: [T, vocab], zeros for tokens that do not count."""
    _, lse = head_loss(x, w, targets, scale)
    on = counts(targets, len(w))
    at = np.nonzero(on)[0]
    r = np.zeros((len(x), len(w)))
    r[at] = np.exp(logits(np.asarray(x)[at], w, scale) - lse[at, None])
    r[at, np.asarray(targets, dtype=np.int64)[at]] -= 1.0
    return r * (scale * np.asarray(dloss, dtype=np.float64))[:, None]


def head_backward(x, w, targets, dloss, scale):
    """(dx, dw)"""
    r = head_slope(x, w, targets, dloss, scale)
    on = counts(targets, len(w))
    return r @ np.asarray(w, dtype=np.float64), r[on].T @ np.asarray(x, dtype=np.float64)[on]


def newton_schulz(g, steps, a, b, c, eps):
    """X and |X|_F of the first and after every step, on the smaller side."""
    x = np.asarray(g, dtype=np.float64)
    x = x / (np.sqrt((x * x).sum()) + eps)
    norms = [np.linalg.norm(x)]
    tall = x.shape[0] > x.shape[1]
    x = x.T if tall else x
    for _ in range(steps):
        gram = x @ x.T
        x = a * x + (b * gram + c * (gram @ gram)) @ x
        norms.append(np.linalg.norm(x))
    return (x.T if tall else x), norms
