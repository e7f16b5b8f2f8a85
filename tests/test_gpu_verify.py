"""Verification of drafted tokens on the GPU against the float64 oracle: accepted
counts and tokens exactly."""
import numpy as np
import pytest

from oracle import verify as ov
from tests.gpu_common import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def rgd():
    import paper_2607_20791_amd as m
    return m


def _run(rgd, target, draft, tokens, n_draft, T, min_p, u):
    t = torch()
    S, K1, V = target.shape
    dev = lambda a, dt: t.from_numpy(np.ascontiguousarray(a, dtype=dt)).cuda()  # noqa: E731
    out = t.full((S, K1), -9, dtype=t.int32, device="cuda")
    cnt = t.full((S,), -9, dtype=t.int32, device="cuda")
    ws = t.empty(rgd.verify_workspace_bytes(S, K1 - 1, V), dtype=t.uint8, device="cuda").fill_(255)
    rgd.verify_drafts(dev(target, np.float32), None if draft is None else dev(draft, np.float32), dev(tokens, np.int32),
                      None if n_draft is None else dev(n_draft, np.int32), T, min_p, dev(u, np.float32), ws, out, cnt)
    t.cuda.synchronize()
    return out.cpu().numpy(), cnt.cpu().numpy()


def _compare(rgd, target, draft, tokens, n_draft, T, min_p, u):
    T, min_p = float(np.float32(T)), float(np.float32(min_p))
    got, cnt = _run(rgd, target, draft, tokens, n_draft, T, min_p, u)
    S, K1, _ = target.shape
    for s in range(S):
        want, n = ov.verify(target[s], None if draft is None else draft[s], tokens[s],
                            K1 - 1 if n_draft is None else n_draft[s], T, min_p, u[s])
        assert cnt[s] == n and got[s].tolist() == want.tolist(), (s, cnt[s], n, got[s], want)
    return cnt


def _inputs(seed, S, K, V, T=1.0, near=0.5, scale=2.0, min_p=0.0):
    """Logits of a target and of a model near it, drafts drawn from the latter's truncated distribution."""
    r = np.random.default_rng(seed)
    target = (r.standard_normal((S, K + 1, V)) * scale).astype(np.float32)
    for s in range(S):
        for i in range(K + 1):
            at = r.integers(0, V, 5)
            target[s, i, at] += r.random(5).astype(np.float32) * 8
    draft = (target[:, :K] + near * r.standard_normal((S, K, V))).astype(np.float32)
    gumbel = -np.log(-np.log(r.random((S, K, V)) + 1e-300))
    low = draft.max(-1, keepdims=True) + T * np.log(min_p) if min_p > 0 else -np.inf
    tokens = np.argmax(np.where(draft >= low, draft / max(T, 1e-3) + gumbel * (T > 0), -np.inf), -1)
    u = (r.integers(0, 1 << 24, (S, K + 1)) / float(1 << 24)).astype(np.float32)
    return target, draft, tokens, u


@pytest.mark.parametrize("V", [2, 5, 127, 1000, 4095, 4096, 4097, 8193, 50257])
@pytest.mark.parametrize("T,min_p", [(1.0, 0.1), (2.0, 0.0), (0.7, 0.3), (0.0, 0.1), (1.0, 1.0)])
def test_against_the_oracle(rgd, V, T, min_p):
    S, K = (6, 4) if V < 9000 else (3, 2)
    target, draft, tokens, u = _inputs(V + int(T * 10), S, K, V, T, min_p=min_p)
    counts = _compare(rgd, target, draft, tokens, None, T, min_p, u)
    assert V < 1000 or T == 0 or min_p == 1 or counts.max() > 0
    _compare(rgd, target, None, target[:, :K].argmax(-1), None, T, min_p, u)


@pytest.mark.parametrize("V", [262144, 262145, 1 << 20])
def test_the_largest_vocabularies(rgd, V):
    for T, min_p in ((1.0, 0.05), (0.0, 0.0), (2.0, 0.0)):
        target, draft, tokens, u = _inputs(V % 1000, 2, 1, V, T, min_p=min_p)
        _compare(rgd, target, draft, tokens, None, T, min_p, u)


@pytest.mark.parametrize("V", [63, 64, 65, 255, 256, 257, 2047, 2048, 2049, 8191, 8192, 16385])
def test_vocabularies_at_the_borders_of_what_a_wave_reads(rgd, V):
    for T, min_p in ((1.0, 0.05), (1.5, 0.0), (0.0, 0.0)):
        target, draft, tokens, u = _inputs(V, 5, 3, V, T, min_p=min_p)
        _compare(rgd, target, draft, tokens, [3, 0, 1, 2, 3], T, min_p, u)
        target[:, :, -3:] += 12  # what is kept lies at the row's end, a NaN among it
        target[:, :, -2] = np.nan
        _compare(rgd, target, draft, tokens, None, T, min_p, u)
        _compare(rgd, target, None, np.full((5, 3), V - 1), None, T, min_p, u)


def test_logits_beyond_32_bits(rgd):
    """More than 2^31 logits: the last sequence's draws, the others without drafts."""
    t = torch()
    S, K, V = 20, 110, 1 << 20
    assert S * (K + 1) * V > 2**31
    target, draft, tokens, u = _inputs(5, 1, 3, V, 1.0, min_p=0.05)
    z, x = t.zeros(S, K + 1, V, device="cuda"), t.zeros(S, K, dtype=t.int32, device="cuda")
    z[-1, :4] = t.from_numpy(target[0]).cuda()
    x[-1, :3] = t.from_numpy(tokens[0].astype(np.int32)).cuda()
    nd = t.zeros(S, dtype=t.int32, device="cuda")
    nd[-1] = 3
    us = t.full((S, K + 1), 0.5, device="cuda")
    us[-1, :3], us[-1, K] = t.from_numpy(u[0, :3]).cuda(), float(u[0, 3])
    out, cnt = (t.empty(*s, dtype=t.int32, device="cuda") for s in ((S, K + 1), (S,)))
    ws = t.empty(rgd.verify_workspace_bytes(S, K, V), dtype=t.uint8, device="cuda")
    rgd.verify_drafts(z, None, x, nd, 1.0, float(np.float32(0.05)), us, ws, out, cnt)
    want, n = ov.verify(target[0], None, tokens[0], 3, 1.0, float(np.float32(0.05)), u[0])
    assert int(cnt[-1]) == n and out[-1, :4].tolist() == want.tolist()
    assert bool((cnt[:-1] == 0).all()) and bool((out[:-1, 0] == V // 2).all())  # equal logits: half of the ids


@pytest.mark.parametrize("S", [12, 60, 100])
def test_rows_in_parts_of_every_size(rgd, S):
    """Few rows are summed in small parts, many in larger ones; with min-p and with every id kept."""
    for T, min_p in ((1.0, 0.05), (3.0, 0.0)):
        target, draft, tokens, u = _inputs(S, S, 2, 50257, T, min_p=min_p)
        _compare(rgd, target, draft, tokens, None, T, min_p, u)


def test_ragged_counts_and_tokens_outside(rgd):
    target, draft, tokens, u = _inputs(3, 9, 5, 777)
    n = [0, 1, 2, 3, 4, 5, -4, 99, 5]
    tokens[4, 1], tokens[5, 0], tokens[8, 3] = -1, 777, 2**31 - 1
    for d in (draft, None):
        _compare(rgd, target, d, tokens, n, 1.0, 0.05, u)


def test_many_sequences_and_one_draft(rgd):
    target, draft, tokens, u = _inputs(4, 300, 1, 260)
    c = _compare(rgd, target, draft, tokens, None, 1.5, 0.02, u)
    assert 0 < c.sum() < 300


def test_many_drafts(rgd):
    target, draft, tokens, u = _inputs(5, 2, 255, 300, near=0.05)
    c = _compare(rgd, target, draft, tokens, None, 1.0, 0.0, u)
    assert c.max() > 5


def test_a_flat_row_of_many_ids(rgd):
    """Every id kept, no weight stands out: the draw needs every running sum."""
    target, draft, tokens, u = _inputs(6, 8, 2, 152064, scale=0.1, near=0.1)
    for T, min_p in ((1.0, 0.0), (3.0, 0.05)):
        _compare(rgd, target, draft, tokens, None, T, min_p, u)


@pytest.mark.parametrize("T", [0.0, 1.0])
def test_masked_ids_and_rows_without_a_distribution(rgd, T):
    target, draft, tokens, u = _inputs(7, 8, 3, 5000, T)
    target[0, :, 100:4900] = -np.inf          # a grammar's mask
    draft[0, :, 100:4900] = -np.inf
    target[1, 1] = -np.inf                    # nothing left
    target[2, 0] = np.nan
    target[3, 2, 17] = np.inf
    target[4, :, ::3] = np.nan                # NaN counts as -inf
    draft[5, 0] = -np.inf                     # a draft row without a distribution
    draft[5, 1, 9] = np.inf
    target[6] = np.finfo(np.float32).min      # all at the type's lowest value
    target[7, 0, 1:] = -np.inf                # one id has everything
    tokens[0], tokens[7, 0] = target[0, :3].argmax(-1), 0
    _compare(rgd, target, draft, tokens, None, T, 0.1, u)
    _compare(rgd, target, None, tokens, None, T, 0.0, u)


def test_exact_borders(rgd):
    """Two equal halves and quarters: u on the border refuses, and draws the next id."""
    target = np.full((4, 2, 8), -np.inf, np.float32)
    target[:2, :, [2, 5]] = 0.0
    target[2:, :, [0, 3, 4, 7]] = 1.0
    u = np.array([[0.5, 0.5], [0.49999997, 0.0], [0.25, 0.5], [0.0, 0.75]], np.float32)
    got, cnt = _run(rgd, target, None, [[2], [2], [3], [7]], None, 1.0, 0.0, u)
    assert cnt.tolist() == [0, 1, 0, 1]
    assert got.tolist() == [[5, -1], [2, 2], [4, -1], [7, 7]]
    # identical rows: every draft is kept whatever u is, and a kept token's share is the target's
    z = np.random.default_rng(0).standard_normal((3, 3, 4100)).astype(np.float32)
    tok = z[:, :2].argmax(-1)
    got, cnt = _run(rgd, z, z[:, :2], tok, None, 1.0, 0.0, np.full((3, 3), 1 - 2.0**-24, np.float32))
    assert (cnt == 2).all() and (got[:, :2] == tok).all()


def test_ties_at_zero_temperature_go_to_the_lowest_id(rgd):
    z = np.zeros((1, 3, 9000), np.float32)
    z[0, 0, [50, 8000]] = 3.0
    z[0, 1, [4097, 4096]] = 2.0
    got, cnt = _run(rgd, z, None, [[50, 4097]], None, 0.0, 0.0, np.zeros((1, 3)))
    assert cnt.tolist() == [1] and got[0].tolist() == [50, 4096, -1]


def test_temperatures_at_the_ends(rgd):
    target, draft, tokens, u = _inputs(8, 4, 2, 3000)
    for T in (1e-30, 1e-6, 1e6, 1e38):
        _compare(rgd, target, draft, target[:, :2].argmax(-1), None, T, 0.1, u)


def test_a_captured_call_replays(rgd):
    t = torch()
    target, draft, tokens, u = _inputs(9, 5, 3, 6001)
    dev = [t.from_numpy(np.ascontiguousarray(a)).cuda() for a in (target, draft, tokens.astype(np.int32), u)]
    ws = t.empty(rgd.verify_workspace_bytes(5, 3, 6001), dtype=t.uint8, device="cuda")
    out, cnt = t.zeros(5, 4, dtype=t.int32, device="cuda"), t.zeros(5, dtype=t.int32, device="cuda")

    def call():
        rgd.verify_drafts(dev[0], dev[1], dev[2], None, 1.0, 0.05, dev[3], ws, out, cnt)

    t.cuda.synchronize()
    graph = t.cuda.CUDAGraph()
    with t.cuda.graph(graph):
        call()
    for turn in range(4):
        dev[3].copy_(t.from_numpy(np.roll(u, turn, 0)))
        graph.replay()
        t.cuda.synchronize()
        got = out.clone(), cnt.clone()
        call()
        t.cuda.synchronize()
        assert t.equal(out, got[0]) and t.equal(cnt, got[1])


def test_binding_refuses_wrong_tensors(rgd):
    t = torch()
    z = t.zeros(2, 4, 10, device="cuda")
    tok, u = t.zeros(2, 3, dtype=t.int32, device="cuda"), t.zeros(2, 4, device="cuda")
    out, cnt = t.zeros(2, 4, dtype=t.int32, device="cuda"), t.zeros(2, dtype=t.int32, device="cuda")
    ws = t.empty(rgd.verify_workspace_bytes(2, 3, 10), dtype=t.uint8, device="cuda")
    good = [z, None, tok, None, 1.0, 0.1, u, ws, out, cnt]
    rgd.verify_drafts(*good)
    for i, bad in ((0, z.double()), (0, z[:, :, ::2]), (0, z.cpu()), (1, z), (2, tok.long()), (2, tok[:, :2]), (3, tok),
                   (4, -1.0), (5, 2.0), (6, u[:, :3]), (7, ws[:8]), (8, tok), (9, tok)):
        with pytest.raises(rgd.RGDError) as e:
            rgd.verify_drafts(*(good[:i] + [bad] + good[i + 1:]))
        assert e.value.code == 1


@pytest.mark.parametrize("V", [1000, 20011])
@pytest.mark.parametrize("T,min_p", [(1.0, 0.1), (1.0, 0.0), (0.7, 0.05), (2.5, 0.0)])
def test_a_refused_draft_of_equal_rows_draws_from_the_target(rgd, V, T, min_p):
    """p - q is 0 everywhere: a draft outside the vocabulary, or one that the truncation leaves out, is refused and
    the token comes from p itself."""
    S, K = 8, 2
    target, _, tokens, u = _inputs(V, S, K, V, T)
    draft = target[:, :K].copy()
    tokens[:, 1] = [-1, V, -1, 2**31 - 1, -2**31, V + 5, -1, V]
    if min_p > 0:
        tokens[::2, 0] = target[::2, 0].argmin(-1)  # p = q = 0
        tokens[1::2, 0] = target[1::2, 0].argmax(-1)
    counts = _compare(rgd, target, draft, tokens, None, T, min_p, u)
    assert counts.tolist() == ([0, 1] * 4 if min_p > 0 else [1] * 8)
