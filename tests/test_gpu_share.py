"""Shared pages and the attention over them on the GPU against the float64 oracle."""
import numpy as np
import pytest

from oracle import paged as op
from tests.gpu_common import torch
from tests.test_gpu_paged import Case, _dt, _i32, _np

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def rgd():
    import paper_2607_20791_amd as m
    return m


def _forks(rgd, roots, branches, tails, new, stale=float("nan"), width=0, spare=3, shuffle=True, **kw):
    """Prompts of the given lengths, each with `branches` sequences that share its whole pages, in shuffled slots: branch j
    ends tails[j] positions behind its prompt.  Slots without a position are `stale`.  Returns the case and labels."""
    t = torch()
    ps = kw.get("ps", 16)
    S = len(roots) * branches
    pages = [[] for _ in range(S)]
    lens = np.zeros(S, int)
    at = 0
    for p, L in enumerate(roots):
        whole = list(range(at, at + L // ps))
        at += L // ps
        for j in range(branches):
            s = p * branches + j
            lens[s] = L + tails[s % len(tails)]
            own = op.used_pages(lens[s], ps) - len(whole)
            pages[s] = whole + list(range(at, at + own))
            at += own
    x = Case(rgd, S, max(width, max(len(p) for p in pages), 1), at + spare, **kw)
    to = x.r.permutation(x.n_pages)
    order = x.r.permutation(S) if shuffle else np.arange(S)
    mask = t.ones(x.n_pages, ps, dtype=t.bool)
    for slot, s in enumerate(order):
        x.pages[slot, :len(pages[s])] = to[pages[s]]
        x.lens[slot] = lens[s]
        for j, p in enumerate(x.pages[slot, :len(pages[s])]):
            x.refs[p] += 1
            mask[p, :min(ps, lens[s] - j * ps)] = False
    x.c.pages.copy_(_i32(x.pages))
    x.c.lens.copy_(_i32(x.lens))
    x.c.refs.copy_(_i32(x.refs))
    mask = mask.cuda()
    x.c.pool_k.masked_fill_(mask[None, :, None, :, None], stale)
    x.c.pool_v.masked_fill_(mask[None, :, None, None, :], stale)
    x.new = np.array([new[s % len(new)] for s in order])
    return x, np.array([s // branches for s in order])


def _plan(x, n, new, heads, group):
    t, rgd = torch(), x.rgd
    plan = t.empty(rgd.paged_share_bytes(x.c, n, heads), dtype=t.uint8, device="cuda").fill_(255)
    shared = t.full((x.S,), -7, dtype=t.int32, device="cuda")
    rgd.paged_share(x.c, n, None if new is None else _i32(new), heads, None if group is None else _i32(group), plan, shared)
    t.cuda.synchronize()
    m = np.full(x.S, n) if new is None else np.clip(new, 0, n)
    want = op.share(x.c.pages.cpu().numpy(), x.c.lens.cpu().numpy(), x.ps, m, group)
    assert np.array_equal(shared.cpu().numpy(), want)
    return plan, want


def _attend(x, layer, heads, n, new, group, spread=1.0, lse=True, stride=0, check=True):
    """Runs plan and attention and compares every row; returns the outputs and what is shared."""
    t, rgd = torch(), x.rgd
    S, d = x.S, x.d
    plan, shared = _plan(x, n, new, heads, group)
    q = t.from_numpy(x.r.standard_normal((S * n, heads * d + stride), dtype=np.float32) * spread).cuda().to(_dt(x.bf16))
    q = q[:, :heads * d].unflatten(1, (heads, d))
    out = t.full((S * n, heads * d), 7.0, dtype=_dt(x.bf16), device="cuda")
    ls = t.full((S * n, heads), 7.0, device="cuda") if lse else None
    ws = t.empty(rgd.paged_attention_shared_workspace_bytes(x.c, n, heads), dtype=t.uint8, device="cuda").fill_(255)
    rgd.paged_attention_shared(x.c, layer, q, n, plan, ws, out, ls)
    t.cuda.synchronize()
    if check:
        compare(x, layer, heads, n, new, q, out, ls)
    return q, out, ls, shared, plan, ws


def compare(x, layer, heads, n, new, q, out, ls):
    S, d = x.S, x.d
    o, l, qn = _np(out).reshape(S, n, heads, d), _np(ls).reshape(S, n, heads) if ls is not None else None, _np(q).reshape(S, n, heads, d)
    pages, lens = x.c.pages.cpu().numpy(), np.clip(x.c.lens.cpu().numpy(), 0, x.width * x.ps)
    pk, pv = _np(x.c.pool_k)[layer], _np(x.c.pool_v)[layer]
    for s in range(S):
        m = n if new is None else min(max(int(new[s]), 0), n)
        assert (o[s, m:] == 7).all() and (l is None or (l[s, m:] == 7).all())
        k, v, there = op.gather(pk, pv, pages[s], int(lens[s]), x.ps)
        ro, rl = op.attention(qn[s, :m], k, v, there, int(lens[s]) - m)
        N = int(lens[s])
        if not m or not there.any():
            assert (o[s, :m] == 0).all() and (l is None or np.isneginf(l[s, :m]).all())
            continue
        # as for the attention without sharing: a score is summed in d + 4 roundings of at most 2^-24 of sum |q k|; its
        # error reaches a weight twice; the hardware exponential adds 2^-22, weights held as two bf16 2^-16, sums over N
        # positions N roundings, and the joins of up to 64 pieces 64 more; the output is rounded once
        mag = np.abs(qn[s, :m]).sum(-1).max() * np.abs(k[there]).max() / np.sqrt(d)
        score = (d + 4) * 2.0**-24 * mag + 2.0**-22 * mag
        half = 2.0**-8 if x.bf16 else 2.0**-24
        tol = half * np.abs(ro) + (2 * score + 2.0**-15 * x.bf16 + 2.0**-21 + 2 * (N + 64) * 2.0**-24) * np.abs(v[there]).max()
        assert (np.abs(o[s, :m] - ro) <= tol).all(), (s, np.abs(o[s, :m] - ro).max(), tol.min())
        if l is not None:
            fin = np.isfinite(rl)
            assert (np.isneginf(l[s, :m]) == ~fin).all()
            bound = score + (N + 64) * 2.0**-24 + 2.0**-20 + 2.0**-22 * np.abs(rl[fin])
            assert (np.abs(l[s, :m][fin] - rl[fin]) <= bound).all(), (s, np.abs(l[s, :m][fin] - rl[fin]).max())


def test_plans_of_random_tables(rgd):
    for seed in range(30):
        r = np.random.default_rng(seed)
        S, width, ps = int(r.integers(1, 40)), int(r.integers(1, 9)), int(r.choice([16, 32]))
        x = Case(rgd, S, width, 12, ps=ps, hk=1, d=32, seed=seed)
        x.pages = np.where(r.random((S, width)) < 0.85, np.arange(width), r.integers(-2, 14, (S, width)))
        x.c.pages.copy_(_i32(x.pages))
        x.c.lens.copy_(_i32(r.integers(-5, width * ps + 9, S)))
        n = int(r.integers(1, 20))
        for group in (None, np.zeros(S, int), r.integers(-2, S + 2, S), r.integers(0, 3, S) % S):
            _plan(x, n, r.integers(-1, n + 3, S), 4, group)
            _plan(x, n, None, 4, group)


@pytest.mark.parametrize("S", [255, 256, 257, 1100])
def test_plans_of_many_sequences(rgd, S):
    r = np.random.default_rng(S)
    x = Case(rgd, S, 7, 20, hk=1, d=32, seed=1)
    x.pages = np.where(r.random((S, 7)) < 0.98, np.arange(7), 9)
    x.c.pages.copy_(_i32(x.pages))
    x.c.lens.copy_(_i32(r.integers(0, 113, S)))
    _plan(x, 3, r.integers(0, 4, S), 2, r.integers(0, 40, S))
    _plan(x, 3, None, 2, None)


def test_plans_of_long_tables(rgd):
    x = Case(rgd, 5, 3000, 4000, hk=1, d=32, seed=2)
    x.pages[:] = np.arange(3000)
    x.pages[3, 2500], x.pages[4, 1023] = 3999, 3998
    x.c.pages.copy_(_i32(x.pages))
    x.c.lens.copy_(_i32([48000, 47000, 46000, 48000, 48000]))
    for group in (None, [0, 0, 0, 0, 1], [0, 0, 1, 1, 2], [3, 1, 1, 3, 4]):
        _plan(x, 1, None, 2, None if group is None else np.array(group))


TAILS = [1, 2, 15, 16, 17, 33, 5, 64, 70]


@pytest.mark.parametrize("bf16", [True, False])
@pytest.mark.parametrize("d", [32, 64, 128])
@pytest.mark.parametrize("hk,G", [(1, 1), (2, 4), (1, 16), (2, 3)])
def test_forks_of_prompts(rgd, bf16, d, hk, G):
    x, group = _forks(rgd, [100, 17, 48, 300], 5, TAILS, [1], hk=hk, d=d, bf16=bf16, seed=d + G)
    _, _, _, shared, _, _ = _attend(x, 1, hk * G, 1, None, group, spread=2.0)
    assert sorted(set(shared)) == [16, 48, 96, 288]


@pytest.mark.parametrize("bf16", [True, False])
@pytest.mark.parametrize("n,hk,G,d,ps,branches", [(2, 2, 4, 64, 16, 3), (5, 2, 4, 128, 32, 7), (9, 1, 2, 32, 48, 2),
                                                  (17, 2, 1, 64, 16, 4), (5, 1, 8, 128, 64, 16), (70, 1, 2, 64, 16, 3)])
def test_several_tokens(rgd, bf16, n, hk, G, d, ps, branches):
    tails = [n + t for t in (0, 3, 16, 40)]
    x, group = _forks(rgd, [4 * ps + 5, 9 * ps], branches, tails, [n, n - 1, 1, 0], hk=hk, d=d, ps=ps, bf16=bf16, seed=n)
    _attend(x, 0, hk * G, n, x.new, group, spread=1.5, stride=64)


@pytest.mark.parametrize("bf16", [True, False])
@pytest.mark.parametrize("root,branches", [(3000, 2), (4097, 33), (2000, 64)])
def test_long_prompts(rgd, bf16, root, branches):
    x, group = _forks(rgd, [root], branches, [1, 7, 40], [1], hk=2, d=128, bf16=bf16, seed=root, layers=1)
    _, _, _, shared, _, _ = _attend(x, 0, 8, 1, None, None, spread=1.0)
    assert (shared == root // 16 * 16).all()


def test_many_prompts_of_every_length(rgd):
    roots = [16 * k + k % 16 for k in range(40)]
    x, group = _forks(rgd, roots, 3, TAILS, [1], hk=2, d=64, seed=3)
    _attend(x, 1, 8, 1, None, group)


@pytest.mark.parametrize("bf16", [True, False])
def test_sequences_that_share_nothing(rgd, bf16):
    """Labels that say otherwise, groups of one, empty sequences and slots without new tokens."""
    x, group = _forks(rgd, [40, 0, 90, 200, 16, 8], 2, [3, 20], [1, 2, 0, 2, 1], hk=2, d=64, bf16=bf16, seed=4)
    one = np.arange(x.S)
    whole = _attend(x, 1, 8, 2, x.new, np.zeros(x.S, int))[3]
    alone = _attend(x, 1, 8, 2, x.new, one)[3]
    assert not whole.any() and not alone.any()
    _attend(x, 1, 8, 2, x.new, -one - 1)
    x.c.lens[0] = 0
    _attend(x, 1, 8, 2, x.new, group)
    _attend(x, 1, 8, 2, np.zeros(x.S, int), group)


def test_groups_of_different_kinds_at_once(rgd):
    x, group = _forks(rgd, [700, 33, 0, 160, 320], 6, [1, 4, 30], [1, 0, 2, 3], hk=2, d=128, seed=5)
    group[::7] = -1          # by themselves, though their pages are shared
    group[3::11] = x.S + 5
    _attend(x, 1, 8, 3, x.new, group)


@pytest.mark.parametrize("bf16", [True, False])
def test_bad_pages_are_masked_for_all(rgd, bf16):
    """A page outside the pool among the shared ones, among a branch's own, and a whole shared part of such pages."""
    x, group = _forks(rgd, [100, 64, 48], 4, [1, 20, 33], [1], hk=2, d=64, bf16=bf16, seed=6)
    for s in range(x.S):
        if group[s] == 0:
            x.pages[s, 2] = -1
        if group[s] == 1:
            x.pages[s, :4] = 10**6
    x.pages[0, x.lens[0] // 16] = -3
    x.c.pages.copy_(_i32(x.pages))
    _attend(x, 1, 8, 1, None, group)


@pytest.mark.parametrize("bf16", [True, False])
@pytest.mark.parametrize("value", [float("inf"), float("-inf"), float("nan")])
def test_a_shared_value_that_is_not_finite_stays_in_its_dimension(rgd, bf16, value):
    x, group = _forks(rgd, [200, 100], 3, [1, 9], [1], hk=2, d=64, bf16=bf16, seed=7)
    q, clean, _, shared, plan, ws = _attend(x, 0, 8, 1, None, group)
    s = int(np.flatnonzero(group == 0)[0])
    p = int(x.pages[s, 3])
    x.c.pool_v[0, p, 1, 20, 5] = value
    t = torch()
    out = t.zeros_like(clean)
    x.rgd.paged_attention_shared(x.c, 0, q, 1, plan, ws, out)
    got, want = _np(out).reshape(x.S, 2, 4, 64), _np(clean).reshape(x.S, 2, 4, 64)
    hit = np.zeros_like(got, bool)
    hit[group == 0, 1, :, 20] = True
    assert np.array_equal(got[~hit], want[~hit])
    # an infinity times the two parts of a weight, one of which may be negative, may also leave NaN
    assert not np.isfinite(got[hit]).any()


@pytest.mark.parametrize("bf16", [True, False])
def test_scores_far_apart(rgd, bf16):
    """Weights of the shared part of 2^-100 of a branch's own, and the other way round."""
    x, group = _forks(rgd, [160], 4, [1, 20], [1], hk=1, d=64, bf16=bf16, seed=8)
    for big in (0, 1):
        x.c.pool_k.copy_(torch().where(torch().isnan(x.c.pool_k), x.c.pool_k, 0.01))
        shared_pages = [int(p) for p in x.pages[0, :10]]
        own = sorted({int(p) for row in x.pages for p in row if p >= 0} - set(shared_pages))
        x.c.pool_k[:, shared_pages if big else own] *= 300.0
        _attend(x, 0, 4, 1, None, group, spread=2.0)


def test_a_plan_of_other_sizes_writes_nothing(rgd):
    t = torch()
    x, group = _forks(rgd, [100, 64], 4, [5, 20], [2], hk=2, d=64, seed=9)
    big = t.empty(rgd.paged_share_bytes(x.c, 4, 16), dtype=t.uint8, device="cuda")
    q = t.randn(2 * x.S, 8, 64, device="cuda").bfloat16()
    ws = t.empty(rgd.paged_attention_shared_workspace_bytes(x.c, 2, 8), dtype=t.uint8, device="cuda")
    out, lse = t.full((2 * x.S, 512), 7.0, device="cuda").bfloat16(), t.full((2 * x.S, 8), 7.0, device="cuda")
    for fill in ("zeros", "other n", "other heads"):
        big.zero_()
        if fill != "zeros":
            rgd.paged_share(x.c, 4 if fill == "other n" else 2, None, 8 if fill == "other n" else 4, _i32(group), big)
        rgd.paged_attention_shared(x.c, 0, q, 2, big, ws, out, lse)
        t.cuda.synchronize()
        assert (out == 7).all() and (lse == 7).all(), fill


def test_bits_repeat_and_a_group_of_one_is_the_plain_attention(rgd):
    t = torch()
    x, group = _forks(rgd, [500, 333], 5, [3, 30, 8], [1], hk=2, d=128, seed=10)
    q, out, lse, _, plan, ws = _attend(x, 0, 8, 1, None, group)
    for _ in range(3):
        ws.fill_(x.r.integers(0, 255))
        again, l2 = t.zeros_like(out), t.zeros_like(lse)
        x.rgd.paged_attention_shared(x.c, 0, q, 1, plan, ws, again, l2)
        assert t.equal(again, out) and t.equal(l2, lse)
    alone, _ = _plan(x, 1, None, 8, np.arange(x.S))
    x.rgd.paged_attention_shared(x.c, 0, q, 1, alone, ws, again, l2)
    plain, l3 = t.zeros_like(out), t.zeros_like(lse)
    pws = t.empty(rgd.paged_attention_workspace_bytes(x.c, 1, 8), dtype=t.uint8, device="cuda")
    rgd.paged_attention(x.c, 0, q, 1, None, pws, plain, l3)
    assert float((again.float() - plain.float()).abs().max()) <= 2.0**-7 * float(plain.float().abs().max())
    assert float((l2 - l3).abs().max()) <= 1e-5


def test_a_table_wider_than_its_sequences(rgd):
    x, group = _forks(rgd, [100, 64], 4, [5, 20], [1], hk=2, d=64, seed=11, width=5000)
    _attend(x, 1, 8, 1, None, group)


def test_offsets_beyond_32_bits(rgd):
    t = torch()
    n_pages, ps, d = 1 << 19, 16, 128
    pages = np.array([[n_pages - 1, n_pages - 2, n_pages - 3 - s] for s in range(4)])
    c = rgd.PagedCache(t.zeros(2, n_pages, 1, ps, d, dtype=t.bfloat16, device="cuda"), t.zeros(2, n_pages, 1, d, ps, dtype=t.bfloat16, device="cuda"),
                       _i32(pages), _i32([40, 41, 42, 43]), t.zeros(n_pages, dtype=t.int32, device="cuda"), _i32([0]))
    for p in set(pages.ravel()):
        c.pool_k[1, p] = t.randn(1, ps, d, device="cuda").bfloat16()
        c.pool_v[1, p] = t.randn(1, d, ps, device="cuda").bfloat16()
    q = t.randn(4, 4, d, device="cuda").bfloat16()
    plan = t.empty(rgd.paged_share_bytes(c, 1, 4), dtype=t.uint8, device="cuda")
    ws = t.empty(rgd.paged_attention_shared_workspace_bytes(c, 1, 4), dtype=t.uint8, device="cuda")
    out = t.zeros(4, 4 * d, dtype=t.bfloat16, device="cuda")
    rgd.paged_share(c, 1, None, 4, None, plan)
    rgd.paged_attention_shared(c, 1, q, 1, plan, ws, out)
    for s in range(4):
        k = t.cat([c.pool_k[1, int(p), 0] for p in pages[s]])[:40 + s].double()
        v = t.cat([c.pool_v[1, int(p), 0].T for p in pages[s]])[:40 + s].double()
        a = t.softmax((q[s].double() @ k.T) / d**0.5, -1) @ v
        assert float((out[s].view(4, d).double() - a).abs().max()) <= 2.0**-8 * float(a.abs().max()) + 1e-3


def test_another_stream_and_a_captured_turn(rgd):
    """Plan and attention of two layers on a side stream, and captured once and replayed while the cache moves on."""
    t = torch()
    x, group = _forks(rgd, [200, 90], 4, [3, 30, 8], [1], hk=2, d=128, seed=12)
    g = _i32(group)
    q = t.randn(2, x.S, 8, 128, device="cuda").bfloat16()
    plan = t.empty(rgd.paged_share_bytes(x.c, 1, 8), dtype=t.uint8, device="cuda")
    ws = t.empty(rgd.paged_attention_shared_workspace_bytes(x.c, 1, 8), dtype=t.uint8, device="cuda")
    out, lse = t.zeros(2, x.S, 1024, device="cuda").bfloat16(), t.zeros(2, x.S, 8, device="cuda")

    def turn():
        rgd.paged_share(x.c, 1, None, 8, g, plan)
        for layer in range(2):
            rgd.paged_attention_shared(x.c, layer, q[layer], 1, plan, ws, out[layer], lse[layer])

    turn()
    t.cuda.synchronize()
    want = (out.clone(), lse.clone())
    out.zero_(), lse.zero_()
    t.cuda.synchronize()
    side = t.cuda.Stream()
    with t.cuda.stream(side):
        turn()
    side.synchronize()
    assert t.equal(out, want[0]) and t.equal(lse, want[1])
    graph = t.cuda.CUDAGraph()
    with t.cuda.graph(graph):
        turn()
    for i in range(4):
        x.c.lens.sub_(1)
        q.mul_(0.9)
        turn()
        t.cuda.synchronize()
        want = (out.clone(), lse.clone())
        out.zero_(), lse.zero_()
        graph.replay()
        t.cuda.synchronize()
        assert t.equal(out, want[0]) and t.equal(lse, want[1])


def test_binding_refuses_wrong_tensors(rgd):
    t = torch()
    x, group = _forks(rgd, [64], 2, [5], [1], hk=2, d=64, seed=13)
    plan = t.empty(rgd.paged_share_bytes(x.c, 1, 8), dtype=t.uint8, device="cuda")
    g, one = _i32(group), _i32([1, 1])
    share = dict(n=1, n_new=one, n_heads=8, group=g, plan=plan, shared=t.empty(2, dtype=t.int32, device="cuda"))
    rgd.paged_share(x.c, **share)
    for kw in (dict(plan=None), dict(plan=plan[:64]), dict(plan=plan.int()), dict(group=g.long()), dict(group=g[:1]), dict(n_new=g.cpu()),
               dict(shared=g.float()), dict(shared=g), dict(n=0), dict(n_heads=3), dict(n=1 << 32), dict(n_heads=1 << 32)):
        with pytest.raises(rgd.RGDError):
            rgd.paged_share(x.c, **{**share, **kw})
    ws = t.empty(rgd.paged_attention_shared_workspace_bytes(x.c, 1, 8), dtype=t.uint8, device="cuda")
    q, out = t.zeros(2, 8, 64, device="cuda").bfloat16(), t.zeros(2, 512, device="cuda").bfloat16()
    good = dict(layer=0, q=q, n=1, plan=plan, workspace=ws, out=out, lse=t.zeros(2, 8, device="cuda"))
    rgd.paged_attention_shared(x.c, **good)
    for kw in (dict(layer=2), dict(layer=1 << 32), dict(q=None), dict(q=q.float()), dict(q=q[:1]), dict(q=q.view(2, 512)), dict(n=2), dict(plan=None),
               dict(plan=plan[:100]), dict(workspace=None), dict(workspace=ws[:8]), dict(out=None), dict(out=out.float()),
               dict(out=q), dict(lse=out), dict(q=q[:, :5])):
        with pytest.raises(rgd.RGDError):
            rgd.paged_attention_shared(x.c, **{**good, **kw})


@pytest.mark.parametrize("many", [False, True])
@pytest.mark.parametrize("bf16,n,d", [(True, 1, 128), (True, 5, 64), (False, 1, 32), (False, 3, 128)])
def test_own_parts_around_every_length(rgd, bf16, n, d, many):
    """Own parts of whole steps of 32 positions and one more or less, where a wave, a workgroup and the runs take turns; few
    sequences, and as many as do not fit the chip at once."""
    steps = [1, 31, 32, 33, 63, 64, 65, 96, 97, 128, 129, 319, 321, 767, 768, 769, 800]
    hk = 8 if many else 2
    x, group = _forks(rgd, [32 if bf16 else 48] * (7 if many else 1), len(steps), [n + t for t in steps], [n, 1], hk=hk, d=d, bf16=bf16, layers=1,
                      seed=n + d)
    _attend(x, 0, hk * 3, n, x.new, group)


@pytest.mark.parametrize("bf16,n,hk,G,d", [(True, 300, 1, 4, 64), (False, 260, 1, 2, 32), (True, 1024, 1, 1, 32)])
def test_pieces_of_prompts(rgd, bf16, n, hk, G, d):
    x, group = _forks(rgd, [50, 33], 2, [n, n + 9], [n, n - 7, 1, n], hk=hk, d=d, bf16=bf16, layers=1, seed=n)
    _attend(x, 0, hk * G, n, x.new, group)


def test_two_captured_turns_share_plan_and_workspace(rgd):
    """Graphs of one token and of three, of one cache, over the same plan and workspace, replayed in turn."""
    t = torch()
    x, group = _forks(rgd, [200, 90], 4, [3, 30, 400], [1], hk=2, d=64, seed=13)
    g = _i32(group)
    size = lambda f: max(f(x.c, n, 8) for n in (1, 3))  # noqa: E731
    plan = t.empty(size(rgd.paged_share_bytes), dtype=t.uint8, device="cuda")
    ws = t.empty(size(rgd.paged_attention_shared_workspace_bytes), dtype=t.uint8, device="cuda")
    turns = []
    for n in (1, 3):
        q = t.randn(x.S * n, 8, 64, device="cuda").bfloat16()
        out = t.zeros(x.S * n, 512, device="cuda").bfloat16()

        def turn(n=n, q=q, out=out):
            rgd.paged_share(x.c, n, None, 8, g, plan)
            rgd.paged_attention_shared(x.c, 0, q, n, plan, ws, out)

        turn()
        t.cuda.synchronize()
        want = out.clone()
        graph = t.cuda.CUDAGraph()
        with t.cuda.graph(graph):
            turn()
        turns.append((graph, out, want, q))  # q: the graph reads it
    for i in (0, 1, 1, 0, 1, 0):
        turns[0][1].zero_(), turns[1][1].zero_()
        plan.fill_(255), ws.fill_(255)
        turns[i][0].replay()
        t.cuda.synchronize()
        assert t.equal(turns[i][1], turns[i][2]) and not turns[1 - i][1].any()


@pytest.mark.parametrize("bf16", [True, False])
@pytest.mark.parametrize("hk,G", [(2, 3), (2, 4), (1, 8)])
@pytest.mark.parametrize("width", [0, 400])
def test_memory_that_is_no_plan_writes_nothing(rgd, bf16, hk, G, width):
    """A plan of memory as it comes: floats below 0 are counts whose products with G pass 2^31, and random bytes."""
    t = torch()
    x, group = _forks(rgd, [100, 64], 4, [5, 20], [2], hk=hk, d=64, bf16=bf16, seed=14, width=width)
    plan = t.empty(rgd.paged_share_bytes(x.c, 2, hk * G), dtype=t.uint8, device="cuda")
    words = plan[:plan.numel() // 4 * 4].view(t.int32)
    q = t.randn(2 * x.S, hk * G, 64, device="cuda").to(_dt(bf16))
    ws = t.empty(rgd.paged_attention_shared_workspace_bytes(x.c, 2, hk * G), dtype=t.uint8, device="cuda").fill_(255)
    out, lse = t.full((2 * x.S, hk * G * 64), 7.0, device="cuda").to(_dt(bf16)), t.full((2 * x.S, hk * G), 7.0, device="cuda")
    pool = (x.c.pool_k.clone(), x.c.pool_v.clone())
    for fill in (-10.0, -3.0, -2.5, -1.0, 1e30, None):
        if fill is None:
            plan.copy_(t.from_numpy(x.r.integers(0, 256, plan.numel()).astype(np.uint8)))
        else:
            words.copy_(t.full((words.numel(),), fill, device="cuda").view(t.int32))
        rgd.paged_attention_shared(x.c, 0, q, 2, plan, ws, out, lse)
        t.cuda.synchronize()
        assert (out == 7).all() and (lse == 7).all(), fill
    same = lambda a, b: bool(((a == b) | (t.isnan(a) & t.isnan(b))).all())  # noqa: E731
    assert same(x.c.pool_k, pool[0]) and same(x.c.pool_v, pool[1])


@pytest.mark.parametrize("bf16", [True, False])
@pytest.mark.parametrize("power", [0, 10, 16, 17, 20])
def test_large_scores_of_shared_positions(rgd, bf16, power):
    """Queries and keys of whole numbers, so that products are exact: scores around 2^power (in units of log 2), whose spacing in fp32 is
    2^-4 at the last, and whose distances from the maximum, which is all that a weight depends on, are small."""
    t = torch()
    d, hk, G = 64, 1, 8
    x, group = _forks(rgd, [320, 200], 4, [9, 40, 70], [1], hk=hk, d=d, bf16=bf16, seed=power, layers=1)
    # score = 32768 k0 + 128 k1 + k2 + offset of the head, times log2(e) / 8
    aim = int(round((2.0**power - 4) / (np.log2(np.e) / 8)))
    k = np.zeros((x.n_pages, hk, x.ps, d), np.float32)
    k[..., 0], k[..., 1] = aim // 32768, aim % 32768 // 128
    k[..., 2] = aim % 128 + x.r.integers(-20, 21, k.shape[:-1])
    k[..., 3] = 1
    x.c.pool_k[0] = t.where(t.isnan(x.c.pool_k[0]), x.c.pool_k[0], t.from_numpy(k).cuda().to(_dt(bf16)))
    q = np.zeros((x.S, hk * G, d), np.float32)
    q[..., 0], q[..., 1], q[..., 2] = 32768, 128, 1
    q[..., 3] = np.linspace(-40, 40, hk * G).round()
    q = t.from_numpy(q).cuda().to(_dt(bf16))
    plan, shared = _plan(x, 1, None, hk * G, group)
    assert shared.min() == 192
    out, lse = t.zeros(x.S, hk * G * d, dtype=_dt(bf16), device="cuda"), t.zeros(x.S, hk * G, device="cuda")
    ws = t.empty(rgd.paged_attention_shared_workspace_bytes(x.c, 1, hk * G), dtype=t.uint8, device="cuda").fill_(255)
    rgd.paged_attention_shared(x.c, 0, q, 1, plan, ws, out, lse)
    pages, pk, pv = x.c.pages.cpu().numpy(), _np(x.c.pool_k)[0], _np(x.c.pool_v)[0]
    o, l, qn = _np(out).reshape(x.S, 1, hk * G, d), _np(lse).reshape(x.S, 1, hk * G), _np(q).reshape(x.S, 1, hk * G, d)
    for s in range(x.S):
        N = int(x.lens[s])
        kk, v, there = op.gather(pk, pv, pages[s], N, x.ps)
        ro, rl = op.attention(qn[s], kk, v, there, N - 1)
        # a distance is at most 40 log2(e) / 8 < 8: rounded once, as its factor is, 2^-24 of it each in log2 units, and the
        # exponential 2^-22; of a weight that comes twice into the output.  Two bf16 hold it to 2^-16; sums and joins as elsewhere
        tol = (2.0**-8 if bf16 else 2.0**-24) * np.abs(ro) + (2 * (16 * 2.0**-24 + 2.0**-22) + 2.0**-15 * bf16 + 2 * (N + 64) * 2.0**-24) * np.abs(v).max()
        assert (np.abs(o[s] - ro) <= tol).all(), (s, np.abs(o[s] - ro).max())
        # lse: the maximum and the sum's logarithm are added and brought to base e, three roundings of its size, the maximum's own and its factor's
        assert (np.abs(l[s] - rl) <= 5 * 2.0**-24 * (np.abs(rl) + 16) + (N + 64) * 2.0**-24).all(), (s, np.abs(l[s] - rl).max())
