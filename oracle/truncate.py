"""One draw under temperature, top-k, top-p and min-p in float64, from a given uniform number.

The ids are ordered by logit, equal ones lower id first, and weighted exp((z - max z) / T); each limit keeps a leading part
of what the one before it kept.  The draw is the smallest id whose running kept weight exceeds u times the kept weight.
"""
from __future__ import annotations

from typing import NamedTuple

import numpy as np


class Draw(NamedTuple):
    token: int      # -1: no distribution
    logp: float
    kept: np.ndarray  # ids, in order
    margin: float   # how near u and top_p come to a border, in units of the largest weight


def kept_ids(z, T, top_k=0, top_p=1.0, min_p=0.0):
    """(ids by descending logit, their weights, the distance of top_p's border); z without NaN, finite maximum, T > 0."""
    order = np.argsort(-z, kind="stable")
    w = np.exp((z[order] - z[order[0]]) / T)
    n = int((z > -np.inf).sum())
    if top_k > 0:
        n = min(n, int(top_k))
    margin = np.inf
    if top_p < 1:
        run = np.cumsum(w[:n])
        target = max(top_p, 0.0) * run[-1]
        before = run - w[:n]
        inside = before[1:] < target
        margin = np.abs(before[1:] - target).min() if n > 1 else np.inf
        n = 1 + int(np.argmin(inside)) if not inside.all() else n
    if min_p > 0:
        low = T * np.log(min(min_p, 1.0)) if min_p < 1 else 0.0
        n = min(n, int((z[order] - z[order[0]] >= low).sum()))
    return order[:n], w[:n], margin


def draw(z, u, T=1.0, top_k=0, top_p=1.0, min_p=0.0):
    z = np.asarray(z, np.float64)
    z = np.where(np.isnan(z), -np.inf, z)
    top = z.max()
    if not np.isfinite(top):
        return Draw(-1, -np.inf, np.zeros(0, int), np.inf)
    if not T > 0:
        x = int(np.argmax(z))
        return Draw(x, 0.0, np.array([x]), np.inf)
    top_p, min_p = (1.0 if np.isnan(top_p) else top_p), (0.0 if np.isnan(min_p) else min_p)
    ids, w, margin = kept_ids(z, T, top_k, top_p, min_p)
    order = np.argsort(ids)
    ids, w = ids[order], w[order]
    u = 0.0 if np.isnan(u) else min(max(float(u), 0.0), 1.0 - 2.0**-24)
    run = np.cumsum(w)
    at = int(np.searchsorted(run, u * run[-1], side="right"))
    margin = min(margin, float(np.abs(run[:-1] - u * run[-1]).min()) if len(run) > 1 else np.inf)
    return Draw(int(ids[at]), (z[ids[at]] - top) / T - np.log(w.sum()), ids, margin)
