"""The paged-sequence and draft-verification oracles: reference counts follow the
tables through any run of operations, and verified drafts are distributed as the
target (by summation over every outcome of a small vocabulary)."""
import numpy as np
import pytest

from oracle import paged, verify


def _counts(pages, lens, ps, n):
    refs = np.zeros(n, int)
    for s in range(len(lens)):
        np.add.at(refs, pages[s, :paged.used_pages(lens[s], ps)], 1)
    return refs


@pytest.mark.parametrize("seed", range(5))
def test_counts_follow_the_tables(seed):
    r = np.random.default_rng(seed)
    S, width, ps, n = 6, 5, 4, 14
    pages, lens, refs = np.full((S, width), -1), np.zeros(S, int), np.zeros(n, int)
    refused = 0
    for _ in range(60):
        what = r.integers(3)
        if what == 0:
            pages, lens, refs = paged.select(pages, lens, refs, ps, r.integers(-1, S + 1, S), r.integers(-1, 18, S))
        elif what == 1:
            pages, lens, refs, copies, ok = paged.reserve(pages, lens, refs, ps, r.integers(-1, 6, S))
            refused += not ok
            assert len({t for _, t in copies}) == len(copies)
        else:
            pages, refs, moves, live = paged.compact(pages, lens, refs, ps)
            assert (refs[:live] > 0).all() and (refs[live:] == 0).all()
            assert all(f >= live > t for f, t in moves)
        assert np.array_equal(refs, _counts(pages, lens, ps, n))
        for s in range(S):  # the entries behind a sequence's pages hold nothing
            assert (pages[s, paged.used_pages(lens[s], ps):] == -1).all()
    assert refused


def test_a_swap_and_a_fork_at_once():
    pages = np.array([[3, 1], [2, -1], [-1, -1]])
    lens, refs = np.array([6, 3, 0]), np.array([0, 1, 1, 1, 0])
    p, n, c = paged.select(pages, lens, refs, 4, np.array([1, 0, 0]), np.array([-1, -1, 4]))
    assert p.tolist() == [[2, -1], [3, 1], [3, -1]] and n.tolist() == [3, 6, 4] and c.tolist() == [0, 1, 1, 2, 0]


def test_reserve_copies_a_shared_partial_page():
    pages = np.array([[3, -1], [3, -1]])
    lens, refs = np.array([2, 2]), np.array([0, 0, 0, 2])
    p, n, c, copies, ok = paged.reserve(pages, lens, refs, 4, np.array([0, 3]))
    assert ok and copies == [(3, 0)] and p.tolist() == [[3, -1], [0, 1]] and c.tolist() == [1, 1, 0, 1]


@pytest.mark.parametrize("min_p,T,draft", [(0.0, 1.0, True), (0.3, 0.7, True), (0.1, 2.0, False), (0.0, 0.0, True)])
def test_first_token_is_distributed_as_the_target(min_p, T, draft):
    """P(first token = j) summed over the drafted token, the acceptance and the draw
    equals p_j: the accepted measure of u is min(1, p/q), and the drawn id's measure its weight."""
    r = np.random.default_rng(3)
    V, grid = 5, 2000
    zt, zd = r.normal(size=(2, V)), r.normal(size=(1, V))
    p = verify.distribution(zt[0], T, min_p)
    q = verify.distribution(zd[0], T, min_p) if draft else None
    us = (np.arange(grid) + 0.5) / grid
    got = np.zeros(V)
    for x in range(V):
        weight = q[x] if draft else 1.0 / V  # certain drafts: any order of them
        if weight == 0:
            continue
        acc = np.mean([verify.verify(zt, zd if draft else None, [x], 1, T, min_p, [u, 0.5])[1] for u in us])
        hist = np.zeros(V)
        if acc < 1:
            for u in us:
                hist[verify.verify(zt, zd if draft else None, [x], 1, T, min_p, [1 - 1e-12, u])[0][0]] += 1 / grid
        one = (1 - acc) * hist
        one[x] += acc
        if not draft:  # each drafted token by itself leaves the target's distribution
            assert np.abs(one - p).max() < 4 / grid * V
        got += weight * one
    assert np.abs(got - p).max() < 4 / grid * V


def test_rows_without_a_distribution_and_tokens_outside():
    z = np.zeros((2, 4))
    assert verify.verify(z, None, [9], 1, 1.0, 0.0, [0.0, 0.3])[0].tolist() == [1, -1]
    z[0] = -np.inf
    assert verify.verify(z, None, [1], 1, 1.0, 0.0, [0.0, 0.3])[0].tolist() == [-1, -1]
    z[0] = [np.nan, 0, 0, np.nan]
    assert verify.verify(z, None, [0], 1, 1.0, 0.0, [0.0, 0.6])[0].tolist() == [2, -1]
