"""Paged sequences in float64 / plain integers: page tables with shared pages,
their forks, roll-backs, reservations and compaction, what groups of them share, and causal
attention of a sequence's last tokens over its pages.

Arrays as the library lays them out: pages [S][width], lens [S], refs [n_pages],
pool_k [L][n_pages][Hkv][ps][D], pool_v [L][n_pages][Hkv][D][ps].
"""
from __future__ import annotations

import numpy as np


def used_pages(length, ps):
    return -(-int(length) // ps)


def select(pages, lens, refs, ps, parent=None, keep=None):
    """Sequence s becomes the first min(keep[s], len) positions of parent[s]; returns new arrays."""
    S = len(lens)
    new_pages, new_lens, new_refs = pages.copy(), lens.copy(), refs.copy()
    for s in range(S):
        p = s if parent is None or not 0 <= parent[s] < S else int(parent[s])
        n = int(lens[p])
        if keep is not None and keep[s] >= 0:
            n = min(n, int(keep[s]))
        had, now = used_pages(lens[s], ps), used_pages(n, ps)
        for j in range(had):
            new_refs[pages[s, j]] -= 1
        for j in range(now):
            new_refs[pages[p, j]] += 1
        new_pages[s, :now] = pages[p, :now]
        new_pages[s, now:max(had, now)] = -1
        new_lens[s] = n
    return new_pages, new_lens, new_refs


def reserve(pages, lens, refs, ps, grow):
    """Returns (pages, lens, refs, copies [(from, to)], fits)."""
    S, width = pages.shape
    plan = []
    for s in range(S):
        n, g = int(lens[s]), max(0, int(grow[s]))
        had, now = used_pages(n, ps), used_pages(n + g, ps)
        copy = bool(g > 0 and n % ps and refs[pages[s, had - 1]] > 1)
        plan.append((had, now, copy))
    want = sum(now - had + copy for had, now, copy in plan)
    free = np.flatnonzero(refs == 0)
    if want > len(free) or any(now > width for _, now, _ in plan):
        return pages, lens, refs, [], False
    pages, lens, refs, copies, at = pages.copy(), lens.copy(), refs.copy(), [], 0
    for s, (had, now, copy) in enumerate(plan):
        if copy:
            copies.append((int(pages[s, had - 1]), int(free[at])))
            refs[pages[s, had - 1]] -= 1
            pages[s, had - 1] = free[at]
            refs[free[at]] = 1
            at += 1
        for j in range(had, now):
            pages[s, j] = free[at]
            refs[free[at]] = 1
            at += 1
        lens[s] += max(0, int(grow[s]))
    return pages, lens, refs, copies, True


def compact(pages, lens, refs, ps):
    """Returns (pages, refs, moves [(from, to)], live)."""
    live = int((refs > 0).sum())
    holes = [p for p in range(live) if refs[p] == 0]
    movers = [p for p in range(live, len(refs)) if refs[p] > 0]
    to = {m: h for m, h in zip(movers, holes)}
    pages, refs = pages.copy(), refs.copy()
    for s in range(len(lens)):
        for j in range(used_pages(lens[s], ps)):
            pages[s, j] = to.get(int(pages[s, j]), pages[s, j])
    for m, h in to.items():
        refs[h], refs[m] = refs[m], 0
    return pages, refs, list(to.items()), live


def share(pages, lens, ps, new, group=None):
    """Positions that each sequence with new tokens has, in whole pages in front of them, in common with all others
    of its group that have some; 0 where there is none."""
    S, width = pages.shape
    label = [0] * S if group is None else [int(g) if 0 <= g < S else -1 - s for s, g in enumerate(group)]
    out = np.zeros(S, int)
    for g in set(label):
        members = [s for s in range(S) if label[s] == g and new[s] > 0]
        if len(members) < 2:
            continue
        n = min(max(min(max(int(lens[s]), 0), width * ps) - int(new[s]), 0) // ps for s in members)
        same = [all(pages[s, j] == pages[members[0], j] for s in members) for j in range(n)]
        out[members] = ps * (same.index(False) if False in same else n)
    return out


def gather(pool_k, pool_v, pages_row, length, ps):
    """K and V [length][Hkv][D] of one sequence in one layer; positions on a page outside the pool: masked."""
    n_pages, hk, _, d = pool_k.shape
    k = np.zeros((length, hk, d))
    v = np.zeros((length, hk, d))
    there = np.zeros(length, bool)
    for t in range(length):
        p = int(pages_row[t // ps])
        if 0 <= p < n_pages:
            k[t] = pool_k[p, :, t % ps]
            v[t] = pool_v[p, :, :, t % ps]
            there[t] = True
    return k, v, there


def attention(q, k, v, there, first):
    """q [c][Hq][D]: token i sees positions [0, first + i].  Returns o [c][Hq][D], lse [c][Hq]."""
    c, hq, d = q.shape
    g = hq // k.shape[1]
    o, lse = np.zeros((c, hq, d)), np.full((c, hq), -np.inf)
    for i in range(c):
        n = max(0, first + i + 1)
        seen = there[:n]
        if not seen.any():
            continue
        for h in range(hq):
            a = (k[:n, h // g][seen] @ q[i, h].astype(np.float64)) / np.sqrt(d)
            m = a.max()
            e = np.exp(a - m)
            o[i, h] = e @ v[:n, h // g][seen] / e.sum()
            lse[i, h] = m + np.log(e.sum())
    return o, lse
