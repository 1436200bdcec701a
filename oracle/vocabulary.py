"""fp64 oracle of both ends of a model over a vocabulary, from their definitions
(include/nnconv.h): rows of a table by token number with the table's gradient,
and softmax cross entropy against labels or a teacher's largest logits.

Test infrastructure only: plain numpy, row by row, no code in common with the HIP
library.  Operands are float64 arrays that hold the exact values of the 16-bit
inputs; results are not rounded.
"""
from __future__ import annotations

import numpy as np


def _inside(ids, v):
    return (ids >= 0) & (ids < v)


def embedding_fwd(ids, table, scale):
    y = np.zeros((len(ids), table.shape[1]))
    for r, j in enumerate(ids):
        if 0 <= j < len(table):
            y[r] = scale * table[j]
    return y


def embedding_bwd(ids, dy, v, scale):
    """(gradient before the loss-scale step, sum of the terms' magnitudes, tokens of each row)."""
    d, mag, n = np.zeros((v, dy.shape[1])), np.zeros((v, dy.shape[1])), np.zeros(v, dtype=np.int64)
    for r, j in enumerate(ids):
        if 0 <= j < v:
            d[j] += scale * dy[r]
            mag[j] += abs(scale) * np.abs(dy[r])
            n[j] += 1
    return d, mag, n


def target_shares(targets, teacher, v, scale):
    """q of a row's entries: one share a label, the softmax of the teacher's logits else; zeros in a row
    that does not count."""
    targets = np.asarray(targets)
    rows, k = targets.shape
    q = np.zeros((rows, k))
    for r in range(rows):
        live = _inside(targets[r], v)
        if teacher is not None:
            live &= teacher[r] != -np.inf
        if not live.any():
            continue
        if teacher is None:
            q[r] = live
            continue
        a = scale * teacher[r][live]
        e = np.exp(a - a.max())
        q[r][live] = e / e.sum()
    return q


def cross_entropy(x, w, targets, scale=1.0, teacher=None):
    """Dict of loss, lse, counts (rows that count), p (softmax), z, and dz = p - q, with zeros in rows that do not
    count."""
    targets = np.asarray(targets).reshape(len(x), -1)
    v = len(w)
    q = target_shares(targets, teacher, v, scale)
    counts = _inside(targets, v).any(axis=1) if teacher is None else (_inside(targets, v) & (teacher != -np.inf)).any(axis=1)
    clean = np.where(counts[:, None], x, 0.0)
    z = scale * (clean @ w.T)
    top = z.max(axis=1, keepdims=True)
    lse = (top + np.log(np.exp(z - top).sum(axis=1, keepdims=True)))[:, 0]
    p = np.exp(z - lse[:, None]) * counts[:, None]
    dz, loss = p.copy(), np.zeros(len(x))
    for r in np.nonzero(counts)[0]:
        for i, j in enumerate(targets[r]):
            if q[r, i] == 0.0:
                continue
            dz[r, j] -= q[r, i]
            loss[r] += q[r, i] * (np.log(q[r, i]) + lse[r] - z[r, j])
    return dict(loss=loss, lse=np.where(counts, lse, 0.0), counts=counts, p=p, z=z, dz=dz, q=q, x=clean)


def gradients(o, w, scale, factor):
    """(dx, dw) of factor * sum of the losses, from what cross_entropy gave."""
    return factor * scale * (o["dz"] @ w), factor * scale * (o["dz"].T @ o["x"])
