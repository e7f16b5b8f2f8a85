"""Verification of drafted tokens in float64: the accepted prefix and the token
drawn after it, from given uniforms.

With p the target's and q the draft's truncated distribution (temperature, then
min-p), draft x is accepted while u q(x) < p(x); the first refusal draws from
max(p - q, 0), no refusal from the target's next row.
"""
from __future__ import annotations

import numpy as np


def distribution(z, T, min_p):
    """[V] probabilities; None for a row whose maximum is not finite.  NaN counts as -inf."""
    z = np.asarray(z, np.float64)
    z = np.where(np.isnan(z), -np.inf, z)
    m = z.max()
    if not np.isfinite(m):
        return None
    if T == 0:
        p = np.zeros(len(z))
        p[int(np.argmax(z))] = 1.0
        return p
    x = z - m
    w = np.where(x >= (T * np.log(min_p) if min_p > 0 else -np.inf), np.exp(x / T), 0.0)
    return w / w.sum()


def draw(weights, u):
    c = np.cumsum(weights)
    return int(np.searchsorted(c, u * c[-1], side="right"))


def verify(target, draft, tokens, n_draft, T, min_p, u):
    """target [K+1][V], draft [K][V] or None, tokens [K], u [K+1] -> (out [K+1], accepted)."""
    K = len(tokens)
    V = target.shape[1]
    out = np.full(K + 1, -1, np.int64)
    nd = min(max(int(n_draft), 0), K)
    for i in range(nd + 1):
        p = distribution(target[i], T, min_p)
        rest = p
        if i < nd:
            x = int(tokens[i])
            inside = 0 <= x < V
            if draft is None or T == 0:
                q = np.zeros(V)
                if inside:
                    q[x] = 1.0
            else:
                q = distribution(draft[i], T, min_p)
                q = np.zeros(V) if q is None else q
            if p is not None and inside and float(u[i]) * q[x] < p[x]:
                out[i] = x
                continue
            if p is not None:
                rest = np.maximum(p - q, 0.0)
                rest = rest if rest.sum() > 0 else p
        out[i] = -1 if p is None else draw(rest, float(u[K]))
        return out, i
    raise AssertionError
