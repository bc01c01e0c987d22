"""Definitions in fp64 of the rotation of queries and keys over several position axes, of the norm of their heads in front of it,
and of attention with a sliding window and first tokens that stay visible (numpy, no code of the GPU path)."""
from __future__ import annotations

import numpy as np


def angles(positions, pairs, base, own_frequencies=False):
    """[T, pairs] from positions [axes, T] and the number of pairs of every axis."""
    half, out = sum(pairs), []
    base = float(np.float32(base))
    for axis, n in enumerate(pairs):
        for j in range(n):
            power = j / n if own_frequencies else len(out) / half
            out.append(np.asarray(positions[axis], np.float64) * base ** -power)
    return np.stack(out, axis=1)


def turn(x, a, sign=1.0):
    """x [T, heads, dh]: pairs (i, i + dh/2) turned by sign * a[t, i]."""
    h = x.shape[-1] // 2
    c, s = np.cos(a)[:, None], sign * np.sin(a)[:, None]
    return np.concatenate([x[..., :h] * c - x[..., h:] * s, x[..., h:] * c + x[..., :h] * s], axis=-1)


def rotary_forward(x, a, gain=None, eps=0.0):
    x = np.asarray(x, np.float64)
    if gain is not None:
        x = x / np.sqrt((x * x).mean(-1, keepdims=True) + float(np.float32(eps))) * np.asarray(gain, np.float64)
    return turn(x, a)


def rotary_backward(x, a, dz, gain=None, eps=0.0):
    """(dx, dgain or None)"""
    d = turn(np.asarray(dz, np.float64), a, -1.0)
    if gain is None:
        return d, None
    x, g = np.asarray(x, np.float64), np.asarray(gain, np.float64)
    r = 1.0 / np.sqrt((x * x).mean(-1, keepdims=True) + float(np.float32(eps)))
    n, e = x * r, d * g
    return r * (e - n * (e * n).mean(-1, keepdims=True)), (d * n).sum((0, 1))


def visible(Lq, Lk, window, sinks):
    """[Lq, Lk]: the queries are the sequence's last Lq tokens."""
    p, j = np.arange(Lk - Lq, Lk)[:, None], np.arange(Lk)[None]
    return (j <= p) & ((p - j < window) | (j < sinks))


def probabilities(q, k, window, sinks):
    """(p [Lq, Lk], lse [Lq]) of one head."""
    s = np.where(visible(len(q), len(k), window, sinks), q @ k.T / np.sqrt(q.shape[1]), -np.inf)
    m = s.max(1, keepdims=True) if s.shape[1] else np.zeros((len(q), 1))
    e = np.exp(s - m)
    total = e.sum(1, keepdims=True)
    return e / total, (m + np.log(total))[:, 0]


def attention(q, k, v, window, sinks):
    """One sequence, q [Lq, Hq, dh], k, v [Lk, Hkv, dh] -> o [Lq, Hq, dh], lse [Hq, Lq]."""
    q, k, v = (np.asarray(x, np.float64) for x in (q, k, v))
    group = q.shape[1] // k.shape[1]
    o, lse = np.zeros(q.shape), np.zeros(q.shape[1::-1])
    for h in range(q.shape[1]):
        p, lse[h] = probabilities(q[:, h], k[:, h // group], window, sinks)
        o[:, h] = p @ v[:, h // group]
    return o, lse


def attention_backward(q, k, v, d_o, window, sinks):
    """(dq, dk, dv)"""
    q, k, v, d_o = (np.asarray(x, np.float64) for x in (q, k, v, d_o))
    group, scale = q.shape[1] // k.shape[1], q.shape[2] ** -0.5
    dq, dk, dv = np.zeros(q.shape), np.zeros(k.shape), np.zeros(v.shape)
    for h in range(q.shape[1]):
        n = h // group
        p, _ = probabilities(q[:, h], k[:, n], window, sinks)
        dp = d_o[:, h] @ v[:, n].T
        ds = p * (dp - (p * dp).sum(1, keepdims=True)) * scale
        dq[:, h] = ds @ k[:, n]
        dk[:, n] += ds.T @ q[:, h]
        dv[:, n] += p.T @ d_o[:, h]
    return dq, dk, dv
