"""Definitions in fp64 of the operators at the two ends of a training step (numpy, no code of the GPU path)."""
from __future__ import annotations

import numpy as np


def embedding_forward(table, ids, scale, y):
    """Rows of ``y`` whose id is negative stay as they are; ids past the table give NaN."""
    out = np.array(y, np.float64)
    V = len(table)
    for t, v in enumerate(ids):
        if v >= 0:
            out[t] = scale * np.asarray(table[v], np.float64) if v < V else np.nan
    return out


def embedding_backward(dy, ids, scale, dtable):
    out = np.array(dtable, np.float64)
    for t, v in enumerate(ids):
        if 0 <= v < len(out):
            out[v] += scale * np.asarray(dy[t], np.float64)
    return out


def cross_entropy(logits, labels, weight=None):
    """(loss [T], dlogits [T, V])."""
    T, V = logits.shape
    loss, grad = np.zeros(T), np.zeros((T, V))
    for t in range(T):
        if labels[t] < 0:
            continue
        z = np.asarray(logits[t], np.float64)
        w = 1.0 if weight is None else float(weight[t])
        if labels[t] >= V:
            loss[t], grad[t] = np.nan, np.nan
            continue
        with np.errstate(invalid="ignore", divide="ignore", over="ignore"):
            m = z.max()
            e = np.exp(z - m)
            loss[t] = w * (m + np.log(e.sum()) - z[labels[t]])
            p = e / e.sum()
        p[labels[t]] -= 1.0
        grad[t] = w * p
    return loss, grad


def orthogonalize(G, coefficients, steps, eps):
    """Every step's X as well, the result last: [X0, X1, ...] with as many rows as G's smaller side."""
    a, b, c = (float(np.float32(v)) for v in coefficients)
    X = np.asarray(G, np.float64)
    if X.shape[0] > X.shape[1]:
        X = X.T
    X = X / (np.sqrt((X * X).sum()) + float(np.float32(eps)))
    out = [X]
    for _ in range(steps):
        A = X @ X.T
        X = a * X + (b * A + c * A @ A) @ X
        out.append(X)
    return out
