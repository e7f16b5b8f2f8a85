"""Paged sequences on the GPU against the float64 oracle: page operators (tables,
counts, lengths and pool contents exactly), the append, and attention at the
sizes, masks and layouts where it can go wrong."""
import numpy as np
import pytest

from oracle import paged as op
from tests.gpu_common import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def rgd():
    import paper_2607_20791_amd as m
    return m


def _dt(bf16):
    return torch().bfloat16 if bf16 else torch().float32


def _i32(a):
    return torch().from_numpy(np.ascontiguousarray(a, dtype=np.int32)).cuda()


def _np(t):
    return t.double().cpu().numpy()


class Case:
    """A cache on the GPU and what the oracle holds of it."""

    def __init__(self, rgd, S, width, n_pages, layers=2, hk=2, d=64, ps=16, bf16=True, seed=0):
        t = torch()
        self.rgd, self.r = rgd, np.random.default_rng(seed)
        g = t.Generator(device="cuda").manual_seed(seed)
        mk = lambda *s: t.randn(*s, generator=g, device="cuda").to(_dt(bf16))  # noqa: E731
        self.pages, self.lens, self.refs = np.full((S, width), -1), np.zeros(S, int), np.zeros(n_pages, int)
        self.c = rgd.PagedCache(mk(layers, n_pages, hk, ps, d), mk(layers, n_pages, hk, d, ps), _i32(self.pages),
                                _i32(self.lens), _i32(self.refs), _i32([0]))
        self.S, self.width, self.hk, self.d, self.ps, self.bf16, self.n_pages = S, width, hk, d, ps, bf16, n_pages
        self.ws = t.empty(rgd.paged_workspace_bytes(self.c), dtype=t.uint8, device="cuda")
        self.pk, self.pv = _np(self.c.pool_k), _np(self.c.pool_v)

    def select(self, parent, keep):
        self.rgd.paged_select(self.c, None if parent is None else _i32(parent), None if keep is None else _i32(keep),
                              self.ws)
        self.pages, self.lens, self.refs = op.select(self.pages, self.lens, self.refs, self.ps, parent, keep)

    def reserve(self, grow):
        self.rgd.paged_reserve(self.c, _i32(grow), self.ws)
        self.pages, self.lens, self.refs, copies, ok = op.reserve(self.pages, self.lens, self.refs, self.ps, grow)
        for a, b in copies:
            self.pk[:, b], self.pv[:, b] = self.pk[:, a].copy(), self.pv[:, a].copy()
        return ok

    def compact(self):
        live = _i32([-1])
        self.rgd.paged_compact(self.c, live, self.ws)
        self.pages, self.refs, moves, n = op.compact(self.pages, self.lens, self.refs, self.ps)
        for a, b in moves:
            self.pk[:, b], self.pv[:, b] = self.pk[:, a], self.pv[:, a]
        assert int(live[0]) == n
        return len(moves)

    def append(self, layer, n, new, stride=0):
        """Random rows, in a buffer whose rows lie `stride` elements further apart."""
        t = torch()
        w = self.hk * self.d
        kv = t.from_numpy(self.r.standard_normal((2, self.S * n, w + stride), dtype=np.float32)).cuda().to(_dt(self.bf16))
        k, v = (kv[i, :, :w].view(self.S * n, self.hk, self.d) for i in (0, 1))
        self.rgd.paged_append(self.c, layer, k, v, n, None if new is None else _i32(new))
        k, v = _np(k), _np(v)
        for s in range(self.S):
            m = n if new is None else min(max(int(new[s]), 0), n)
            for i in range(m):
                pos = int(self.lens[s]) - m + i
                if pos >= 0:
                    p = self.pages[s, pos // self.ps]
                    self.pk[layer, p, :, pos % self.ps] = k[s * n + i]
                    self.pv[layer, p, :, :, pos % self.ps] = v[s * n + i]

    def check(self):
        torch().cuda.synchronize()
        got = [y.cpu().numpy() for y in (self.c.pages, self.c.lens, self.c.refs)] + [_np(self.c.pool_k), _np(self.c.pool_v)]
        for name, a, b in zip(("pages", "lens", "refs", "pool_k", "pool_v"), got,
                              (self.pages, self.lens, self.refs, self.pk, self.pv)):
            differ = np.argwhere(a != b)
            assert not len(differ), (name, len(differ), differ[:3].tolist())


@pytest.mark.parametrize("seed,S,width,n_pages,ps,d,bf16", [
    (0, 1, 1, 1, 16, 32, True), (1, 5, 3, 9, 16, 64, False), (2, 7, 4, 20, 32, 128, True), (3, 70, 5, 150, 16, 32, True),
    (4, 1100, 2, 1500, 16, 32, True)])
def test_runs_of_page_operators(rgd, seed, S, width, n_pages, ps, d, bf16):
    x = Case(rgd, S, width, n_pages, layers=2, hk=1, d=d, ps=ps, bf16=bf16, seed=seed)
    r, refused, moved, copied = x.r, 0, 0, 0
    for step in range(24):
        what = step % 4
        if what == 0:
            x.select(r.integers(-1, S + 1, S) if step % 8 else None, r.integers(-1, width * ps + 2, S))
        elif what == 2:
            moved += x.compact()
        else:
            before = x.refs.copy()
            grow = r.integers(-2, ps + 2, S) * (r.random(S) < 0.4)
            ok = x.reserve(grow)
            refused += not ok
            copied += int((x.refs < before).sum())
            if ok:  # up to 3 of the positions made; others may share their pages
                x.append(step % 2, 3, np.minimum(grow, 3))
            assert int(x.c.status[0]) == int(refused > 0)
        x.check()
    if S in (5, 7):
        assert moved and copied


def test_reserve_without_room_changes_nothing(rgd):
    x = Case(rgd, 3, 2, 4)
    assert x.reserve([16, 16, 16])
    x.check()
    assert not x.reserve([1, 1, 0])          # one free page, two wanted
    x.check()
    assert int(x.c.status[0]) == 1
    x.c.status.zero_()
    assert not x.reserve([17, 0, 0])         # more than a table holds
    x.check()
    assert int(x.c.status[0]) == 1
    x.c.status.zero_()
    assert x.reserve([0, 16, 0]) and int(x.c.status[0]) == 0
    x.check()
    assert not x.reserve([2**31 - 1, 0, 0])  # a sum past 32 bits
    x.check()


def test_a_long_table_and_a_large_pool(rgd):
    """More pages than one pass of the planning workgroup, reserved at once and given back."""
    x = Case(rgd, 3, 3000, 5000, layers=1, hk=1, d=32, seed=7)
    assert x.reserve([16 * 2000 + 3, 5, 16 * 1500])
    x.check()
    x.select([2, 1, 0], [16 * 1100, -1, 16 * 1900])
    x.check()
    assert x.reserve([1, 20, 9])
    x.compact()
    x.check()


@pytest.mark.parametrize("hk,d,ps,bf16", [(5, 128, 48, True), (8, 128, 16, True), (3, 64, 64, False)])
def test_pages_of_many_bytes_are_copied_and_moved(rgd, hk, d, ps, bf16):
    """Pages of one and several rounds of a workgroup's copies, and of a part of one."""
    x = Case(rgd, 4, 3, 14, layers=3, hk=hk, d=d, ps=ps, bf16=bf16, seed=hk)
    assert x.reserve([ps + 5, 0, 2 * ps, 3])
    x.append(1, 7, None)
    x.select([0, 0, 0, 3], None)
    assert x.reserve([4, 1, ps, 0])
    x.check()
    x.select(None, [0, -1, 1, -1])
    assert x.compact() > 0
    x.check()


@pytest.mark.parametrize("bf16,d,ps,hk,stride", [(True, 32, 16, 3, 0), (True, 64, 32, 2, 16), (True, 128, 16, 8, 4096),
                                                 (False, 32, 16, 1, 8), (False, 64, 48, 2, 0), (False, 128, 16, 4, 128),
                                                 (True, 128, 4096, 1, 0)])
@pytest.mark.parametrize("n", [1, 7, 70])
def test_append(rgd, bf16, d, ps, hk, stride, n):
    x = Case(rgd, 4, max(1, 160 // ps) + 1, 4 * (160 // ps + 2), hk=hk, d=d, ps=ps, bf16=bf16, seed=n)
    assert x.reserve([70, 85, 1, 100])
    x.append(1, n, [n, max(1, n // 2), 1, n + 5], stride)
    x.check()
    x.append(0, n, None, stride)   # n of each: positions before 0 are left out
    x.check()


def test_append_leaves_out_bad_pages(rgd):
    x = Case(rgd, 2, 2, 4)
    assert x.reserve([20, 20])
    before = x.c.pool_k.clone(), x.c.pool_v.clone()
    x.c.pages.copy_(_i32([[-1, 4], [2**30, -2**31]]))
    k = torch().ones(40, 2, 64, dtype=torch().bfloat16, device="cuda")
    rgd.paged_append(x.c, 0, k, k, 20, None)
    torch().cuda.synchronize()
    assert torch().equal(before[0], x.c.pool_k) and torch().equal(before[1], x.c.pool_v)


# ---------------------------------------------------------------- attention --
def _attention(x, layer, heads, n, new, spread=1.0, lse=True, stride=0):
    """Runs it and compares every row; returns the outputs."""
    t = torch()
    S, d = x.S, x.d
    q = t.from_numpy(x.r.standard_normal((S * n, heads * d + stride), dtype=np.float32) * spread).cuda().to(_dt(x.bf16))
    q = q[:, :heads * d].view(S * n, heads, d) if not stride else q[:, :heads * d].unflatten(1, (heads, d))
    out = t.full((S * n, heads * d), 7.0, dtype=_dt(x.bf16), device="cuda")
    ls = t.full((S * n, heads), 7.0, device="cuda") if lse else None
    ws = t.empty(x.rgd.paged_attention_workspace_bytes(x.c, n, heads), dtype=t.uint8, device="cuda").fill_(255)
    x.rgd.paged_attention(x.c, layer, q, n, None if new is None else _i32(new), ws, out, ls)
    t.cuda.synchronize()
    o, l, qn = _np(out).reshape(S, n, heads, d), _np(ls).reshape(S, n, heads) if lse else None, _np(q).reshape(S, n, heads, d)
    pages, lens = x.c.pages.cpu().numpy(), np.clip(x.c.lens.cpu().numpy(), 0, x.width * x.ps)
    pk, pv = _np(x.c.pool_k)[layer], _np(x.c.pool_v)[layer]
    for s in range(S):
        m = n if new is None else min(max(int(new[s]), 0), n)
        assert (o[s, m:] == 7).all() and (not lse or (l[s, m:] == 7).all())
        k, v, there = op.gather(pk, pv, pages[s], int(lens[s]), x.ps)
        ro, rl = op.attention(qn[s, :m], k, v, there, int(lens[s]) - m)
        # a score's products are exact in fp32 or rounded once, summed in fp32: d + 4 roundings of at most 2^-24 of
        # sum |q k|; the weights follow with that error twice (top and own), the hardware exponential adds 2^-22 and
        # weights held as two bf16 2^-16; sums over N positions N roundings, numerator and denominator; the output is
        # rounded once
        N = int(lens[s])
        if not m or not there.any():
            assert (o[s, :m] == 0).all() and (not lse or np.isneginf(l[s, :m]).all())
            continue
        mag = np.abs(qn[s, :m]).sum(-1).max() * np.abs(k[there]).max() / np.sqrt(d)
        score = (d + 4) * 2.0**-24 * mag + 2.0**-22 * mag
        vmax = np.abs(v[there]).max()
        half = 2.0**-8 if x.bf16 else 2.0**-24
        tol = half * np.abs(ro) + (2 * score + 2.0**-15 * x.bf16 + 2.0**-21 + 2 * (N + 64) * 2.0**-24) * vmax
        assert (np.abs(o[s, :m] - ro) <= tol).all(), (s, np.abs(o[s, :m] - ro).max(), tol.min())
        if lse:
            fin = np.isfinite(rl)
            assert (np.isneginf(l[s, :m]) == ~fin).all()
            bound = score + (N + 64) * 2.0**-24 + 2.0**-20 + 2.0**-22 * np.abs(rl[fin])
            assert (np.abs(l[s, :m][fin] - rl[fin]) <= bound).all(), (s, np.abs(l[s, :m][fin] - rl[fin]).max())
    return out, ls


def _filled(rgd, lens, stale=float("nan"), **kw):
    """Sequences of the given lengths in scattered pages; every slot without a position is `stale`."""
    t = torch()
    ps = kw.get("ps", 16)
    used = [op.used_pages(n, ps) for n in lens]
    x = Case(rgd, len(lens), max(1, max(used)), sum(used) + 2, **kw)
    order = x.r.permutation(x.n_pages)
    at = 0
    mask = t.ones(x.n_pages, ps, dtype=t.bool)
    for s, n in enumerate(lens):
        x.pages[s, :used[s]] = order[at:at + used[s]]
        at += used[s]
        for j in range(used[s]):
            mask[x.pages[s, j], :min(ps, n - j * ps)] = False
    x.lens = np.array(lens)
    x.c.pages.copy_(_i32(x.pages))
    x.c.lens.copy_(_i32(x.lens))
    mask = mask.cuda()
    x.c.pool_k.masked_fill_(mask[None, :, None, :, None], stale)
    x.c.pool_v.masked_fill_(mask[None, :, None, None, :], stale)
    return x


LENS = [0, 1, 15, 16, 17, 31, 32, 33, 47, 63, 64, 65, 127, 129, 255, 256, 257, 300]


@pytest.mark.parametrize("bf16", [True, False])
@pytest.mark.parametrize("d", [32, 64, 128])
@pytest.mark.parametrize("hk,G", [(1, 1), (2, 4), (1, 16), (2, 8)])
def test_attention_at_every_kind_of_length(rgd, bf16, d, hk, G):
    x = _filled(rgd, LENS, hk=hk, d=d, bf16=bf16, seed=d + G)
    _attention(x, 1, hk * G, 1, None, spread=2.0)


@pytest.mark.parametrize("bf16", [True, False])
@pytest.mark.parametrize("n,hk,G,d,ps", [(2, 2, 4, 64, 16), (5, 2, 4, 128, 32), (9, 1, 2, 32, 48), (17, 2, 1, 64, 16),
                                         (5, 1, 24, 128, 16), (33, 1, 8, 64, 64), (3, 3, 5, 32, 16)])
def test_attention_of_several_tokens(rgd, bf16, n, hk, G, d, ps):
    lens = [0, 1, 2, 5, 16, 33, 64, 100, 190]
    x = _filled(rgd, lens, hk=hk, d=d, ps=ps, bf16=bf16, seed=n)
    _attention(x, 0, hk * G, n, None)                                       # more tokens than positions: rows of nothing
    _attention(x, 1, hk * G, n, [0, 1, n, 2, n + 9, -3, n, 1, n - 1], stride=16)


@pytest.mark.parametrize("bf16", [True, False])
@pytest.mark.parametrize("d", [32, 64, 128])
@pytest.mark.parametrize("ps,n", [(32, 1), (64, 1), (48, 6), (16, 16), (64, 16)])
def test_attention_at_every_page_size(rgd, bf16, d, ps, n):
    """One, two and four query tiles over pages of one and several rounds."""
    x = _filled(rgd, [0, 1, 31, 33, 63, 65, 129, 200, 400], hk=2, d=d, ps=ps, bf16=bf16, seed=ps + n)
    _attention(x, 1, 8, n, None)


@pytest.mark.parametrize("bf16", [True, False])
def test_attention_splits_a_long_sequence(rgd, bf16):
    x = _filled(rgd, [3001, 1, 0, 1500], hk=1, d=64, bf16=bf16, seed=5)
    _attention(x, 1, 4, 1, None, spread=3.0)
    _attention(x, 0, 4, 3, [3, 1, 2, 2], lse=False)


@pytest.mark.parametrize("n", [1, 3])
def test_attention_of_many_sequences(rgd, n):
    """More sequences than a wave has lanes, in an uneven order."""
    r = np.random.default_rng(n)
    lens = (r.integers(0, 70, 700) * (r.random(700) < 0.6)).tolist() + [1200, 0, 3]
    x = _filled(rgd, lens, hk=1, d=32, layers=1, seed=n)
    _attention(x, 0, 2, n, None if n == 1 else r.integers(-1, 5, len(lens)))


def test_attention_repeats_its_bits_and_does_not_need_a_clean_workspace(rgd):
    x = _filled(rgd, [700, 3, 64, 0, 1999], hk=2, d=128, seed=9)
    t = torch()
    q = t.randn(5, 8, 128, device="cuda").bfloat16()
    ws = t.empty(rgd.paged_attention_workspace_bytes(x.c, 1, 8), dtype=t.uint8, device="cuda")
    first = None
    for fill in (0, 255, 1):
        ws.fill_(fill)
        out, lse = t.zeros(5, 1024, dtype=t.bfloat16, device="cuda"), t.zeros(5, 8, device="cuda")
        rgd.paged_attention(x.c, 0, q, 1, None, ws, out, lse)
        if first is None:
            first = out, lse
        assert t.equal(out, first[0]) and t.equal(lse, first[1])


@pytest.mark.parametrize("stale", [float("inf"), float("-inf"), 3.0e38])
@pytest.mark.parametrize("bf16", [True, False])
def test_attention_never_reads_what_is_masked(rgd, bf16, stale):
    x = _filled(rgd, LENS, stale=stale, hk=2, d=64, bf16=bf16, seed=3)
    _attention(x, 0, 4, 2, None)


def test_attention_masks_bad_pages_and_clamps_lengths(rgd):
    x = _filled(rgd, [100, 100, 40, 64], hk=1, d=64, seed=4)
    pages = x.c.pages.cpu().numpy()
    pages[0, 2], pages[0, 4], pages[1, :], pages[3, 0] = -1, x.n_pages, 2**31 - 1, -2**31
    x.c.pages.copy_(_i32(pages))
    x.c.lens.copy_(_i32([100, 100, -7, 64]))
    _attention(x, 0, 4, 2, None)
    y = _filled(rgd, [112, 32], hk=1, d=64, seed=6)
    y.c.lens.copy_(_i32([2**31 - 1, 32]))  # the table holds 112
    _attention(y, 0, 4, 1, None)


@pytest.mark.parametrize("bf16", [True, False])
def test_scores_far_apart_and_a_nan(rgd, bf16):
    x = _filled(rgd, [200, 90], hk=1, d=64, bf16=bf16, seed=8)
    x.c.pool_k.mul_(30.0)  # scores of hundreds: one position has everything
    _attention(x, 0, 4, 1, None)
    x.c.pool_k[:, int(x.c.pages[1, 2]), :, 5] = float("nan")  # a visible key of sequence 1
    t = torch()
    q = t.randn(2, 4, 64, device="cuda").to(_dt(bf16))
    ws = t.empty(rgd.paged_attention_workspace_bytes(x.c, 1, 4), dtype=t.uint8, device="cuda")
    out = t.zeros(2, 256, dtype=_dt(bf16), device="cuda")
    rgd.paged_attention(x.c, 0, q, 1, None, ws, out)
    assert bool(t.isfinite(out[0]).all()) and bool(t.isnan(out[1]).all())


@pytest.mark.parametrize("bf16", [True, False])
@pytest.mark.parametrize("n,hk,G,d", [(3, 2, 4, 64), (7, 1, 4, 128), (16, 1, 4, 128), (12, 1, 5, 32)])
def test_later_tokens_do_not_reach_earlier_ones(rgd, bf16, n, hk, G, d):
    """Keys and values that are not finite at a new token's position: the tokens before it get the bits they
    get without them, the others what the formula gives."""
    t = torch()
    lens = [n, 45, 64, 200]
    x = _filled(rgd, lens, hk=hk, d=d, bf16=bf16, seed=n)
    ref, _ = _attention(x, 0, hk * G, n, None)
    q = t.randn(4 * n, hk * G, d, device="cuda").to(_dt(bf16))
    ws = t.empty(rgd.paged_attention_workspace_bytes(x.c, n, hk * G), dtype=t.uint8, device="cuda")

    def run():
        out = t.zeros(4 * n, hk * G * d, dtype=_dt(bf16), device="cuda")
        rgd.paged_attention(x.c, 0, q, n, None, ws, out)
        return out.view(4, n, hk, G, d)

    ref = run()
    inf, nan = float("inf"), float("nan")
    for s, (i, what) in enumerate(((n - 1, (nan, 0)), (n - 2, (inf, 1)), (1, (-inf, 1)), (n // 2, (nan, 1)))):
        pos = lens[s] - n + i
        page = int(x.pages[s, pos // 16])
        if what[1]:
            x.c.pool_v[0, page, 0, 3, pos % 16] = what[0]   # dimension 3 of KV head 0
        else:
            x.c.pool_k[0, page, 0, pos % 16] = what[0]
        got = run()
        assert t.equal(got[s, :i], ref[s, :i]), (s, i)
        assert t.equal(got[:, :, 1:], ref[:, :, 1:])
        late = got[s, i:, 0].float()
        if not what[1]:
            assert bool(t.isnan(late).all())
        else:
            rest = [e for e in range(d) if e != 3]
            assert t.equal(got[s, i:, 0][..., rest], ref[s, i:, 0][..., rest])
            assert bool((t.isnan(late[..., 3]) if what[0] != what[0] else late[..., 3] == what[0]).all())


@pytest.mark.parametrize("bf16", [True, False])
@pytest.mark.parametrize("n,hk,G,d", [(1, 2, 4, 64), (5, 1, 4, 128), (16, 1, 4, 32)])
def test_an_old_value_that_is_not_finite_stays_in_its_dimension(rgd, bf16, n, hk, G, d):
    """Values long before the new tokens, which all of them see: the dimension is not finite, everything else
    keeps its bits."""
    t = torch()
    lens = [300, 700, 90]
    x = _filled(rgd, lens, hk=hk, d=d, bf16=bf16, seed=n)
    q = t.randn(3 * n, hk * G, d, device="cuda").to(_dt(bf16))
    ws = t.empty(rgd.paged_attention_workspace_bytes(x.c, n, hk * G), dtype=t.uint8, device="cuda")

    def run():
        out = t.zeros(3 * n, hk * G * d, dtype=_dt(bf16), device="cuda")
        rgd.paged_attention(x.c, 0, q, n, None, ws, out)
        return out.view(3, n, hk, G, d)

    ref = run()
    for s, (pos, dim, what) in enumerate(((5, 0, float("inf")), (400, 17, float("-inf")), (0, d - 1, float("nan")))):
        x.c.pool_v[0, int(x.pages[s, pos // 16]), 0, dim, pos % 16] = what
        ref[s, :, 0, :, dim] = 0
        got = run()
        assert not bool(t.isfinite(got[s, :, 0, :, dim]).any())
        for i in range(s + 1):
            got[i, :, 0, :, (0, 17, d - 1)[i]] = 0
        assert t.equal(got, ref), s


def test_offsets_beyond_32_bits(rgd):
    """A pool of more than 2^31 elements whose used pages lie at its end."""
    t = torch()
    n_pages, hk, d, ps = 36000, 8, 128, 64
    mk = lambda *s: t.zeros(*s, dtype=t.bfloat16, device="cuda")  # noqa: E731
    assert n_pages * hk * ps * d > 2**31
    small = Case(rgd, 2, 3, 6, layers=1, hk=hk, d=d, ps=ps, seed=1)
    big = rgd.PagedCache(mk(1, n_pages, hk, ps, d), mk(1, n_pages, hk, d, ps), _i32(np.full((2, 3), -1)), _i32([0, 0]),
                         t.ones(n_pages, dtype=t.int32, device="cuda"), _i32([0]))
    big.refs[n_pages - 6:] = 0
    ws = t.empty(rgd.paged_workspace_bytes(big), dtype=t.uint8, device="cuda")
    k, v, q = (t.randn(2 * 150, h, d, device="cuda").bfloat16() for h in (hk, hk, 2 * hk))
    outs = []
    for c, w in ((small.c, small.ws), (big, ws)):
        rgd.paged_reserve(c, _i32([150, 131]), w)
        rgd.paged_append(c, 0, k, v, 150, _i32([150, 131]))
        o = t.zeros(2 * 150, 2 * hk * d, dtype=t.bfloat16, device="cuda")
        rgd.paged_attention(c, 0, q, 150, _i32([150, 131]), t.empty(
            rgd.paged_attention_workspace_bytes(c, 150, 2 * hk), dtype=t.uint8, device="cuda"), o)
        outs.append(o)
    assert int(big.pages.max()) == n_pages - 1 and t.equal(outs[0], outs[1])
    # a shared page at the end is copied there, and the pages move down to the start
    rgd.paged_select(big, _i32([0, 0]), None, ws)
    rgd.paged_reserve(big, _i32([0, 1]), ws)
    big.refs[:n_pages - 6] = 0
    live = _i32([0])
    rgd.paged_compact(big, live, ws)
    assert int(live[0]) == 4 and int(big.pages.max()) == 3
    o = t.zeros_like(outs[0])
    big.lens[1] -= 1
    rgd.paged_attention(big, 0, t.cat([q[:150], q[:150]]), 150, None, t.empty(
        rgd.paged_attention_workspace_bytes(big, 150, 2 * hk), dtype=t.uint8, device="cuda"), o)
    assert t.equal(o[:150], outs[0][:150]) and t.equal(o[150:], outs[0][:150])


# ------------------------------------------------------- as they are used --
def test_branches_grow_fork_roll_back_and_move(rgd):
    """Branches of two prompts over many turns: each turn forks or rolls some back, reserves, appends
    in both layers and attends; the oracle keeps every branch's own history of K and V."""
    S, hk, d = 7, 2, 64
    x = Case(rgd, S, 12, 60, hk=hk, d=d, seed=11)
    r = x.r
    hist = [[np.zeros((0, hk, d)), np.zeros((0, hk, d))] for _ in range(S)]  # layer 0's K and V, by branch
    for turn in range(14):
        if turn:
            parent, keep = np.arange(S), np.full(S, -1)
            for s in r.choice(S, 3, replace=False):
                if r.random() < 0.5:
                    parent[s] = r.integers(S)
                else:
                    keep[s] = r.integers(0, x.lens[s] + 1)
            old = hist
            hist = [[h[:(len(h) if keep[s] < 0 else keep[s])] for h in old[parent[s]]] for s in range(S)]
            x.select(parent, keep)
        n = 40 if turn == 0 else 4
        new = r.integers(0, n + 1, S) if turn else np.array([33, 40, 0, 5, 16, 17, 1])
        assert x.reserve(new)
        x.append(1, n, new)
        x.append(0, n, new)
        for s in range(S):  # what was appended, from the oracle's pool
            for i, (pool, h) in enumerate(zip((x.pk[0], x.pv[0]), hist[s])):
                rows = []
                for pos in range(len(h), len(h) + new[s]):
                    p = x.pages[s, pos // 16]
                    rows.append(pool[p, :, pos % 16] if i == 0 else pool[p, :, :, pos % 16])
                hist[s][i] = np.concatenate([h, np.array(rows).reshape(-1, hk, d)])
        if turn % 5 == 4:
            x.compact()
        x.check()
        # the pool holds each branch's own history, whatever the others did
        for s in range(S):
            k, v, there = op.gather(x.pk[0], x.pv[0], x.pages[s], x.lens[s], 16)
            assert there.all() and np.array_equal(k, hist[s][0]) and np.array_equal(v, hist[s][1])
        _attention(x, 0, 8, n, new)


def test_lse_joins_with_the_shared_prompt(rgd):
    """Attention over a paged tail joined by its log-sum-exp with attention over other positions
    equals attention over both."""
    x = _filled(rgd, [90, 33], hk=2, d=64, bf16=False, seed=13)
    y = _filled(rgd, [57, 33], hk=2, d=64, bf16=False, seed=13)
    z = _filled(rgd, [33, 0], hk=2, d=64, bf16=False, seed=13)
    t = torch()
    for s, (a, b) in enumerate(((57, 33), (33, 0))):  # x: y's positions, then z's
        ky = op.gather(_np(y.c.pool_k)[0], _np(y.c.pool_v)[0], y.pages[s], a, 16)
        kz = op.gather(_np(z.c.pool_k)[0], _np(z.c.pool_v)[0], z.pages[s], b, 16)
        for pos in range(a + b):
            src, i = (ky, pos) if pos < a else (kz, pos - a)
            p = int(x.pages[s, pos // 16])
            x.c.pool_k[0, p, :, pos % 16] = t.from_numpy(src[0][i]).float().cuda()
            x.c.pool_v[0, p, :, :, pos % 16] = t.from_numpy(src[1][i]).float().cuda()
    q = t.randn(2, 4, 64, device="cuda")
    res = []
    for c in (x.c, y.c, z.c):
        ws = t.empty(rgd.paged_attention_workspace_bytes(c, 1, 4), dtype=t.uint8, device="cuda")
        out, lse = t.zeros(2, 256, device="cuda"), t.zeros(2, 4, device="cuda")
        rgd.paged_attention(c, 0, q, 1, None, ws, out, lse)
        res.append((out.double().view(2, 4, 64), lse.double()))
    both = torch().logaddexp(res[1][1], res[2][1])
    joined = sum(o * t.exp(l - both)[..., None] for o, l in res[1:])
    # three attentions, each within the fp32 bound of _attention for N <= 90 at these magnitudes (|q| sum < 80, |k| < 6)
    tol = 3 * (2 * (68 * 2.0**-24 + 2.0**-22) * 80 * 6 / 8 + 2.0**-20 + 2 * 154 * 2.0**-24) * 6
    assert float((joined - res[0][0]).abs().max()) < tol and float((both - res[0][1]).abs().max()) < tol


def test_binding_refuses_wrong_tensors(rgd):
    t = torch()
    x = Case(rgd, 2, 2, 4)
    ok = dict(pool_k=x.c.pool_k, pool_v=x.c.pool_v, pages=x.c.pages, lens=x.c.lens, refs=x.c.refs, status=x.c.status)

    def refused(fn):
        with pytest.raises(rgd.RGDError) as e:
            fn()
        assert e.value.code == 1

    for name, bad in (("pool_k", x.c.pool_k.half()), ("pool_v", x.c.pool_k), ("pool_k", x.c.pool_k[0]),
                      ("pages", x.c.pages.long()), ("lens", x.c.lens[:1]), ("refs", x.c.refs.cpu()),
                      ("pages", x.c.pages[:, ::2]), ("status", x.c.refs)):
        refused(lambda: rgd.PagedCache(**{**ok, name: bad}))
    g = _i32([1, 1])
    refused(lambda: rgd.paged_reserve(x.c, g.long(), x.ws))
    refused(lambda: rgd.paged_reserve(x.c, g[:1], x.ws))
    refused(lambda: rgd.paged_reserve(x.c, g, x.ws[:8]))
    refused(lambda: rgd.paged_select(x.c, g, g.cpu(), x.ws))
    k = t.zeros(2, 2, 64, dtype=t.bfloat16, device="cuda")
    refused(lambda: rgd.paged_append(x.c, 0, k.float(), k, 1))
    refused(lambda: rgd.paged_append(x.c, 0, k, k.transpose(1, 2), 1))
    refused(lambda: rgd.paged_append(x.c, 2, k, k, 1))
    ws = t.empty(rgd.paged_attention_workspace_bytes(x.c, 1, 2), dtype=t.uint8, device="cuda")
    out = t.zeros(2, 128, dtype=t.bfloat16, device="cuda")
    refused(lambda: rgd.paged_attention(x.c, 0, k, 2, None, ws, out))
    refused(lambda: rgd.paged_attention(x.c, 0, k, 1, None, ws, out.float()))
    refused(lambda: rgd.paged_attention(x.c, 0, k[:, :1], 1, None, ws, out[:, :64]))
    refused(lambda: rgd.paged_attention(x.c, 0, k, 1, None, ws, k.view(2, 128)))


def test_another_stream_and_a_captured_turn(rgd):
    """One turn on a side stream, and captured once and replayed: each gives the eager turn's state."""
    t = torch()

    def turn(c, ws, aws, parent, keep, grow, k, v, q, out, lse):
        rgd.paged_select(c, parent, keep, ws)
        rgd.paged_reserve(c, grow, ws)
        rgd.paged_append(c, 0, k, v, 4, grow)
        rgd.paged_attention(c, 0, q, 4, grow, aws, out, lse)

    def state():
        x = Case(rgd, 4, 8, 40, hk=2, d=128, seed=21)
        assert x.reserve([30, 0, 0, 45])
        c = x.c
        r = t.Generator(device="cuda").manual_seed(5)
        mk = lambda *s: t.randn(*s, generator=r, device="cuda").bfloat16()  # noqa: E731
        aws = t.empty(rgd.paged_attention_workspace_bytes(c, 4, 8), dtype=t.uint8, device="cuda")
        out, lse = t.zeros(16, 1024, dtype=t.bfloat16, device="cuda"), t.zeros(16, 8, device="cuda")
        args = (x.ws, aws, _i32([0, 0, 3, 3]), _i32([-1, -1, 33, -1]), _i32([0, 4, 2, 1]), mk(16, 2, 128), mk(16, 2, 128),
                mk(16, 8, 128), out, lse)
        return c, args

    def snapshot(c, args):
        t.cuda.synchronize()
        return [y.clone() for y in (c.pages, c.lens, c.refs, c.pool_k, c.pool_v, args[-2], args[-1])]

    c, args = state()
    eager = []
    for _ in range(4):
        turn(c, *args)
        eager.append(snapshot(c, args))
    c, args = state()
    side = t.cuda.Stream()
    t.cuda.synchronize()
    with t.cuda.stream(side):
        turn(c, *args)
    assert all(t.equal(a, b) for a, b in zip(snapshot(c, args), eager[0]))
    c, args = state()
    t.cuda.synchronize()
    graph = t.cuda.CUDAGraph()
    with t.cuda.graph(graph):
        turn(c, *args)
    noise = t.randn(1000, 1000, device="cuda")
    for want in eager:
        graph.replay()
        assert all(t.equal(a, b) for a, b in zip(snapshot(c, args), want))
        noise = noise @ noise.T / 1000
        t.cuda.synchronize()


@pytest.mark.parametrize("bf16,d", [(True, 32), (False, 128)])
def test_one_workspace_for_every_number_of_tokens(rgd, bf16, d):
    """The workspace for up to n tokens at the most runs there are: smaller counts write nothing behind it."""
    t = torch()
    x = _filled(rgd, [40000, 39000], hk=1, d=d, layers=1, bf16=bf16, seed=2)
    need = x.rgd.paged_attention_workspace_bytes(x.c, 8, 8)
    room = t.full((need + 65536,), 90, dtype=t.uint8, device="cuda")
    for n in (1, 2, 4, 8):
        q = t.randn(2 * n, 8, d, device="cuda").to(_dt(bf16))
        out = [t.zeros(2 * n, 8 * d, dtype=_dt(bf16), device="cuda") for _ in range(2)]
        rgd.paged_attention(x.c, 0, q, n, None, room[:need], out[0])
        rgd.paged_attention(x.c, 0, q, n, None, t.empty_like(room), out[1])
        assert bool((room[need:] == 90).all()), n
        assert t.equal(out[0], out[1]) and bool(t.isfinite(out[0]).all())


@pytest.mark.parametrize("in_place", [False, True])
def test_a_turn_without_room_leaves_the_cache_as_it_is(rgd, in_place):
    """A captured turn (reserve, append, attention, roll-back by what was kept) whose pages run out, with a page
    that two sequences share; later the same turn goes on from where it stood."""
    t = torch()
    x = Case(rgd, 4, 4, 9, layers=1, hk=2, d=64, seed=31)
    assert x.reserve([20, 0, 0, 30])
    x.append(0, 30, [20, 0, 0, 30])
    x.select([0, 0, 2, 3], None)      # 1 shares both pages of 0; four pages held, five free
    x.check()
    c = x.c
    want, grow, kept = _i32([3, 2, 40, 1]), _i32([0, 0, 0, 0]), _i32([2, 2, 39, 1])
    granted = grow if in_place else _i32([7, 7, 7, 7])
    kv, q = t.randn(2, 4 * 40, 2, 64, device="cuda").bfloat16(), t.randn(4 * 40, 4, 64, device="cuda").bfloat16()
    out = t.full((160, 256), 7.0, dtype=t.bfloat16, device="cuda")
    aws = t.empty(rgd.paged_attention_workspace_bytes(c, 40, 4), dtype=t.uint8, device="cuda")

    def turn():
        grow.copy_(want)
        rgd.paged_reserve(c, grow, x.ws, granted)
        rgd.paged_append(c, 0, kv[0], kv[1], 40, granted)
        rgd.paged_attention(c, 0, q, 40, granted, aws, out)
        rgd.paged_select(c, None, c.lens - granted + kept, x.ws)

    t.cuda.synchronize()
    graph = t.cuda.CUDAGraph()
    with t.cuda.graph(graph):
        turn()
    want.copy_(_i32([3, 2, 48, 1]))   # 0 and 1 copy their shared page, 2 wants three pages, 3 has room: five
    graph.replay()
    assert granted.tolist() == [3, 2, 48, 1] and int(c.status[0]) == 0
    assert c.lens.tolist() == [22, 22, 39, 31] and int((c.refs == 0).sum()) == 1
    rgd.paged_select(c, _i32([0, 0, 2, 3]), None, x.ws)   # 0 and 1 share again; two pages are free
    x2 = [y.clone() for y in (c.pages, c.lens, c.refs, c.pool_k, c.pool_v)]
    out.fill_(7.0)
    want.copy_(_i32([3, 2, 20, 1]))   # two copies and a page: three
    for _ in range(3):
        graph.replay()
        assert granted.tolist() == [0] * 4 and int(c.status[0]) == 1
        for a, b in zip((c.pages, c.lens, c.refs, c.pool_k, c.pool_v), x2):
            assert t.equal(a, b)
        assert bool((out == 7).all())
        t.cuda.synchronize()
    rgd.paged_select(c, _i32([0, 0, 2, 3]), _i32([-1, -1, 0, -1]), x.ws)  # 2 is freed
    c.status.zero_()
    want.copy_(_i32([0, 1, -5, 0]))
    pools = c.pool_k.clone(), c.pool_v.clone()
    n0 = int(c.lens[0])
    graph.replay()
    assert granted.tolist() == [0, 1, 0, 0] and int(c.status[0]) == 0
    assert c.lens.tolist() == [n0, n0 + 1, 0, int(x2[1][3])]
    held = int(c.pages[0, n0 // 16])
    assert t.equal(c.pool_k[0, held], pools[0][0, held]) and int(c.pages[1, n0 // 16]) != held


def test_granted_is_what_reserve_gave(rgd):
    """1100 sequences, more than a turn of the planning workgroup."""
    x = Case(rgd, 1100, 2, 1500, layers=1, hk=1, d=32, seed=3)
    granted = _i32(np.full(1100, 9))
    for grow in (x.r.integers(-3, 17, 1100), np.full(1100, 16), x.r.integers(-2, 2, 1100)):
        ok = op.reserve(x.pages, x.lens, x.refs, 16, grow)[-1]
        rgd.paged_reserve(x.c, _i32(grow), x.ws, granted)
        x.pages, x.lens, x.refs = op.reserve(x.pages, x.lens, x.refs, 16, grow)[:3]
        assert granted.tolist() == (np.maximum(grow, 0) * ok).tolist()
        for a, b in ((x.c.pages, x.pages), (x.c.lens, x.lens), (x.c.refs, x.refs)):
            assert np.array_equal(a.cpu().numpy(), b)


@pytest.mark.parametrize("bf16", [True, False])
@pytest.mark.parametrize("n,hk,G,d", [(1, 2, 4, 64), (5, 1, 4, 128), (16, 1, 4, 32)])
def test_values_up_to_the_largest_sum(rgd, bf16, n, hk, G, d):
    """Values whose sum over the positions is just below 2^128, the larger weights behind the smaller ones, by less
    than what moves a running maximum: the output is finite wherever the formula is."""
    t = torch()
    big, lens = 1.6e38, [300, 3000]
    x = _filled(rgd, lens, hk=hk, d=d, layers=1, bf16=bf16, seed=n)
    # a third sequence over one page makes the runs so long that a wave takes several rounds
    pages = np.full((3, 40000), int(x.pages[0, 0]))
    pages[:2, :x.width] = x.pages
    c = rgd.PagedCache(x.c.pool_k, x.c.pool_v, _i32(pages), _i32(lens + [640000]), x.c.refs, x.c.status)
    x.c.pool_k.nan_to_num_(nan=0.0).zero_()
    x.c.pool_v.nan_to_num_(nan=0.0).zero_()
    q = t.zeros(3 * n, hk * G, d, device="cuda", dtype=_dt(bf16))
    q[:, :, 0] = 1.0
    for s, first in enumerate((0, 1500)):  # a wave takes every 64th or 128th position of an item's
        for pos, score in ((first, 0.0), (first + 128, 5.375)):  # 5.375 / ln 2 = 7.75
            p = int(x.pages[s, pos // 16])
            x.c.pool_k[0, p, :, pos % 16, 0] = score * d ** 0.5
            x.c.pool_v[0, p, :, :, pos % 16] = big
    out, lse = t.zeros(3 * n, hk * G * d, dtype=_dt(bf16), device="cuda"), t.zeros(3 * n, hk * G, device="cuda")
    ws = t.empty(rgd.paged_attention_workspace_bytes(c, n, hk * G), dtype=t.uint8, device="cuda")
    rgd.paged_attention(c, 0, q, n, None, ws, out, lse)
    pk, pv, o = _np(x.c.pool_k)[0], _np(x.c.pool_v)[0], _np(out).reshape(3, n, hk * G, d)
    for s, N in enumerate(lens):
        k, v, there = op.gather(pk, pv, x.pages[s], N, 16)
        assert v.sum(0).max() < 2.0**128
        ro, rl = op.attention(_np(q)[s * n:(s + 1) * n], k, v, there, N - n)
        # as in _attention; nothing cancels, so relative to the output itself; one score of one product, at most 5.4
        rel = 2.0**(-8 if bf16 else -24) + 4 * 5.4 * 2.0**-24 + 2.0**-15 * bf16 + 2.0**-21 + 2 * (N + 64) * 2.0**-24
        assert np.isfinite(ro).all() and (np.abs(o[s] - ro) <= rel * ro).all(), (s, np.abs(o[s] / ro - 1).max(), rel)
        assert (np.abs(_np(lse)[s * n:(s + 1) * n] - rl) <= 5.4 * 2.0**-22 + (N + 64) * 2.0**-24 + 2.0**-20 + 2.0**-22 * rl).all()


@pytest.mark.parametrize("bf16", [True, False])
@pytest.mark.parametrize("n,hk,G,d", [(1, 2, 4, 64), (5, 1, 4, 128), (16, 1, 4, 32)])
def test_weights_follow_the_differences_of_large_scores(rgd, bf16, n, hk, G, d):
    """Products of 2^20 and a little, all exact: the weights keep the little."""
    t = torch()
    x = _filled(rgd, [300, 70, 900], hk=hk, d=d, layers=1, bf16=bf16, stale=0.0, seed=n)
    g = t.Generator(device="cuda").manual_seed(n)
    x.c.pool_k.zero_()
    x.c.pool_k[..., 0] = 2.0**20
    x.c.pool_k[..., 1] = t.randint(0, 16, x.c.pool_k.shape[:-1], generator=g, device="cuda").to(_dt(bf16))
    q = t.zeros(3 * n, hk * G, d, device="cuda", dtype=_dt(bf16))
    q[:, :, :2] = 1.0
    out = t.zeros(3 * n, hk * G * d, dtype=_dt(bf16), device="cuda")
    ws = t.empty(rgd.paged_attention_workspace_bytes(x.c, n, hk * G), dtype=t.uint8, device="cuda")
    rgd.paged_attention(x.c, 0, q, n, None, ws, out)
    pk, pv, o = _np(x.c.pool_k)[0], _np(x.c.pool_v)[0], _np(out).reshape(3, n, hk * G, d)
    for s, N in enumerate(x.lens):
        k, v, there = op.gather(pk, pv, x.pages[s], N, 16)
        ro, _ = op.attention(_np(q)[s * n:(s + 1) * n], k, v, there, N - n)
        # a difference is at most 15 / sqrt(d) log2(e) < 4 of the scale, which is rounded twice, and the reference, up
        # to 8 off, so at most 12 rounded to 2^-21; the exponential 2^-22, weights as two bf16 2^-16; numerator and
        # denominator, each with the roundings of its sums
        weight = 12 * 2.0**-23 + 2.0**-21 + 2.0**-22 + 2.0**-16 * bf16
        tol = 2.0**(-8 if bf16 else -24) * np.abs(ro) + (2 * weight + 2 * (N + 64) * 2.0**-24) * np.abs(v).max()
        assert (np.abs(o[s] - ro) <= tol).all(), (s, np.abs(o[s] - ro).max(), tol.max())


def test_roll_back_needs_no_workspace(rgd):
    x = Case(rgd, 3, 3, 9, seed=4)
    assert x.reserve([20, 40, 5])
    for keep in ([17, -1, 0], [16, 3, 9], None):
        rgd.paged_select(x.c, None, None if keep is None else _i32(keep))
        x.pages, x.lens, x.refs = op.select(x.pages, x.lens, x.refs, 16, None, keep)
        x.check()
    for bad in (None, x.ws[:8]):
        with pytest.raises(rgd.RGDError) as e:
            rgd.paged_select(x.c, _i32([0, 0, 0]), None, bad)
        assert e.value.code == 1
    x.check()


@pytest.mark.parametrize("bf16", [True, False])
@pytest.mark.parametrize("n,hk,G,d,ps", [(64, 1, 4, 64, 16), (65, 2, 1, 128, 32), (150, 1, 2, 128, 64), (500, 1, 2, 32, 16),
                                         (1024, 1, 1, 64, 16)])
def test_attention_of_prompt_pieces(rgd, bf16, n, hk, G, d, ps):
    """Many query tiles: whole prompts, pieces behind a prefix, pieces longer than what is there."""
    x = _filled(rgd, [n + 70, n, 0, n // 2 + 1, 40], hk=hk, d=d, ps=ps, layers=1, bf16=bf16, seed=n)
    _attention(x, 0, hk * G, n, [n, n, n, n - 1, 33])


@pytest.mark.parametrize("d", [32, 64, 128])
@pytest.mark.parametrize("n,small", [(1, 1.0), (1, 0.3), (5, 1.0), (16, -0.9)])
def test_small_products_beside_a_large_one(rgd, d, n, small):
    """fp32: two positions, of which one has d - 1 small products beside the 2^24 that both have.  A product passes at most
    d / 4 + 2 additions, each off by half a step of what is there."""
    t = torch()
    from paper_2607_20791_amd import session
    c = session.alloc_paged(1, 1, 1, d, 1, 1, page_size=32, bf16=False)
    c.pages.zero_()
    c.lens.fill_(n + 1)  # every token sees positions 0 and 1; the others weigh nothing
    c.pool_k[0, 0, 0, :, 0] = -2.0**24
    c.pool_k[0, 0, 0, :2, 0] = 2.0**24
    c.pool_k[0, 0, 0, 0, 1:] = small
    c.pool_v[0, 0, 0, :, 0] = 1.0
    ws = t.empty(rgd.paged_attention_workspace_bytes(c, n, 4), dtype=t.uint8, device="cuda")
    out = t.zeros(n, 4 * d, device="cuda")
    rgd.paged_attention(c, 0, t.ones(n, 4, d, device="cuda"), n, None, ws, out)
    w = _np(out)
    x = float(np.float32(small))
    assert ((w > 0) & (w < 1)).all()
    got = np.log(w / (1 - w)) * np.sqrt(d)  # the difference of the two products
    # and four roundings around the weight, which count by its distance from 0 and 1
    bound = (d / 4 + 2) * 2.0**-24 * (2.0**24 + abs(x) * d) + 4 * 2.0**-24 / np.minimum(w, 1 - w) * np.sqrt(d)
    assert (np.abs(got - x * (d - 1)) <= bound).all(), (got.min(), got.max(), x * (d - 1), bound.max())


def test_numbers_beyond_31_bits_are_refused(rgd):
    """They would reach the library as their lowest 32 bits."""
    t = torch()
    x = Case(rgd, 2, 2, 4)
    k = t.zeros(2, 2, 64, dtype=t.bfloat16, device="cuda")
    out = t.zeros(2, 128, dtype=t.bfloat16, device="cuda")
    ws = t.empty(rgd.paged_attention_workspace_bytes(x.c, 1, 2), dtype=t.uint8, device="cuda")
    before = x.c.pool_k.clone()
    for layer in (1 << 32, -(1 << 32), 1 << 31):
        for call in (lambda: rgd.paged_append(x.c, layer, k, k, 1), lambda: rgd.paged_attention(x.c, layer, k, 1, None, ws, out)):
            with pytest.raises(rgd.RGDError) as e:
                call()
            assert e.value.code == 1
    for n, heads in (((1 << 32) + 1, 2), (1, (1 << 32) + 2)):
        with pytest.raises(rgd.RGDError):
            rgd.paged_attention_workspace_bytes(x.c, n, heads)
    assert t.equal(before, x.c.pool_k)


def test_missing_tensors_are_refused(rgd):
    t = torch()
    x = Case(rgd, 2, 2, 4)
    k = t.zeros(2, 2, 64, dtype=t.bfloat16, device="cuda")
    out = t.zeros(2, 128, dtype=t.bfloat16, device="cuda")
    ws = t.empty(rgd.paged_attention_workspace_bytes(x.c, 1, 2), dtype=t.uint8, device="cuda")
    for call in (lambda: rgd.paged_append(x.c, 0, None, k, 1), lambda: rgd.paged_append(x.c, 0, k, None, 1),
                 lambda: rgd.paged_attention(x.c, 0, None, 1, None, ws, out), lambda: rgd.paged_attention(x.c, 0, k, 1, None, ws, None),
                 lambda: rgd.paged_attention(x.c, 0, k, 1, None, None, out), lambda: rgd.paged_reserve(x.c, None, x.ws),
                 lambda: rgd.paged_compact(x.c, None, x.ws),
                 lambda: rgd.verify_drafts(None, None, None, None, 1.0, 0.1, None, None, None, None)):
        with pytest.raises(rgd.RGDError) as e:
            call()
        assert e.value.code == 1
