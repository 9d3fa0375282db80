"""The operators around the beam decode, written out plainly in 64 bits (test infrastructure: only tests/ import this package; the
CUDA path shares no code with it).

* ``norm_rotate``: y = x / sqrt(sum x^2 + eps) or x / sqrt(mean x^2 + eps) * w per head; pairs of the first r elements turned.
* ``delta_rule``: Eq. 1 token by token over ragged sequences, one state per sequence and value head.
* ``sample_row``: softmax with temperature, top-k, top-p, min-p, and the inverse of the running sum at a given uniform number.
"""
from __future__ import annotations

import math

import numpy as np


def norm_rotate(x, norm, eps, scale=1.0, weight=None, positions=None, inv_freq=None, interleaved=False):
    """x [N, H, d] -> fp64 of the same shape."""
    y = np.array(x, dtype=np.float64)
    d = y.shape[-1]
    if norm == "l2":
        y = y / np.sqrt((y * y).sum(-1, keepdims=True) + eps)
    elif norm == "rms":
        y = y / np.sqrt((y * y).sum(-1, keepdims=True) / d + eps)
        if weight is not None:
            y = y * np.asarray(weight, dtype=np.float64)
    if inv_freq is not None:
        f = np.asarray(inv_freq, dtype=np.float64)
        r = 2 * len(f)
        for n, pos in enumerate(positions):
            # an angle in turns, its whole part taken off exactly: position and frequency are dyadic rationals
            for i in range(r // 2):
                angle = math.fmod(float(int(pos)) * float(f[i]), 2 * math.pi)
                c, s = math.cos(angle), math.sin(angle)
                a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + r // 2)
                u, v = y[n, :, a].copy(), y[n, :, b].copy()
                y[n, :, a], y[n, :, b] = u * c - v * s, v * c + u * s
    return y * scale


def delta_rule(q, k, v, alpha, beta, states, ranges, slots, fresh, trace=None):
    """q, k [N, H, dk], v [N, Hv, dv], alpha, beta [N, Hv], states [slots, Hv, dv, dk]; ranges: (first row, one behind the last) per
    sequence; slots[i] < 0: padded.  Returns (out {row: [Hv, dv]}, states), fp64.  trace, a dict: gets per row the norms [Hv] of the state before
    it and of its update vector."""
    q, k, v, alpha, beta = (np.asarray(x, dtype=np.float64) for x in (q, k, v, alpha, beta))
    states = np.array(states, dtype=np.float64)
    g = v.shape[1] // k.shape[1]
    out = {}
    for i, (a, b) in enumerate(ranges):
        if slots[i] < 0:
            continue
        S = np.zeros_like(states[slots[i]]) if fresh[i] else states[slots[i]].copy()
        for t in range(a, b):
            kt, qt = np.repeat(k[t], g, axis=0), np.repeat(q[t], g, axis=0)
            before = np.sqrt((S * S).sum((1, 2)))
            S = S * alpha[t][:, None, None]
            d = beta[t][:, None] * (v[t] - np.einsum("hvk,hk->hv", S, kt))
            if trace is not None:
                trace[t] = (before, np.sqrt((d * d).sum(1)))
            S = S + d[:, :, None] * kt[:, None, :]
            out[t] = np.einsum("hvk,hk->hv", S, qt)
        states[slots[i]] = S
    return out, states


def sample_row(x, u, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0):
    """(token, logprob, how close the draw came to another answer: the distance of uniform * mass to the next border, over the mass)."""
    x = np.array(x, dtype=np.float64)
    x[np.isnan(x)] = -np.inf
    n, best = len(x), x.max()
    if best == -np.inf:
        return -1, -np.inf, 1.0
    order = np.lexsort((np.arange(n), -x))              # descending values, ascending index
    if not temperature > 0:
        return int(order[0]), 0.0, 1.0
    with np.errstate(invalid="ignore"):
        w = np.where(x == best, 1.0, np.where(np.isinf(x), 0.0, np.exp((x - best) / float(temperature))))
    s = w[order]
    count = top_k if 1 <= top_k < n else n
    if top_p < 1:
        before = np.concatenate(([0.0], np.cumsum(s[:count])[:-1]))
        count = max(1, int((before < float(top_p) * math.fsum(s[:count])).sum()))
    keep = np.zeros(n, dtype=bool)
    keep[order[:count]] = True
    if min_p > 0:
        keep &= w >= min(float(min_p), 1.0)
    w = np.where(keep, w, 0.0)
    run = np.cumsum(w)
    u = 0.0 if not u > 0 else min(float(u), 1.0)
    target = u * run[-1]
    token = int(np.searchsorted(run, target, side="right"))
    if token >= n or u >= 1:
        token = int(np.flatnonzero(w)[-1])
    border = np.abs(run - target).min() / run[-1]
    return token, float(np.log(w[token] / run[-1])), float(border)
