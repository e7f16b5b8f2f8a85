"""The append with head norms and rotary positions on the GPU against the float64 oracle."""
import numpy as np
import pytest

from oracle import rotary as orot
from tests.gpu_common import torch
from tests.test_gpu_paged import Case, _dt, _i32, _np

pytestmark = pytest.mark.gpu
U = 2.0**-24  # half a step of fp32


@pytest.fixture(scope="module")
def rgd():
    import paper_2607_20791_amd as m
    return m


def _bound(x, ref, freq, pos, normed, D, bf16, scale):
    """Half a step of the result's type and what fp32 loses before it.  Norm: a sum of D squares in D / 4 + 5 roundings at
    most, of which the root takes half, then division, root and two products: (D / 8 + 7) u of a value.  Angle: the part of a turn is
    rounded to fp32 (at most 1/2, so pi u radians), sine and cosine to 2 u, the factor and two products and a sum to 4 u: 10 u of both
    values of a pair.  In fp64 the turn loses 2^-52 of the position's turns."""
    pair = np.abs(x).max(-1, keepdims=True) * abs(scale) * 2
    far = 2 * np.pi * np.abs(pos * np.abs(freq).max()) * 2.0**-52 if len(freq) else 0.0
    return (2.0**-8 if bf16 else U) * np.abs(ref) * 1.01 + ((D / 8 + 7 if normed else 0) + 10) * U * pair + far * pair + 1e-38


def _run(rgd, x, n, new, dim, interleaved=False, G=2, norms=True, how=None, positions=None, stride=0, in_place=False, eps=1e-5,
         theta=500000.0, scale=1.0, spread=1.0, layer=1):
    t = torch()
    S, hk, D, hq = x.S, x.hk, x.d, x.hk * G
    w = (hq + 2 * hk) * D
    rows = t.from_numpy(x.r.standard_normal((S * n, w + stride), dtype=np.float32) * spread).cuda().to(_dt(x.bf16))
    qkv = rows[:, :w].unflatten(1, (hq + 2 * hk, D))
    q, k, v = qkv[:, :hq], qkv[:, hq:hq + hk], qkv[:, hq + hk:]
    qn, kn, vn, before = _np(q), _np(k), _np(v), rows.clone()
    gains = [t.from_numpy(1 + 0.3 * x.r.standard_normal(D)).float().cuda() for _ in range(2)] if norms else [None, None]
    rot = rgd.Rotary(dim, theta, interleaved, rgd.RotaryScaling(*how) if how else None, scale=scale) if dim else None
    freq, factor = orot.frequencies(dim, theta, *(how or ())) if dim else (np.zeros(0), 1.0)
    factor *= scale
    out = q if in_place else t.full((S * n, hq, D), 7.0, dtype=_dt(x.bf16), device="cuda")
    rgd.paged_append_rotated(x.c, layer, q, k, v, n, rot, out, n_new=None if new is None else _i32(new),
                             positions=None if positions is None else _i32(positions), q_norm=gains[0], k_norm=gains[1], eps=eps)
    t.cuda.synchronize()
    got, pools = _np(out), (_np(x.c.pool_k), _np(x.c.pool_v))
    wk, wv = x.pk.copy(), x.pv.copy()  # what the pools have to hold
    for s in range(S):
        m = n if new is None else min(max(int(new[s]), 0), n)
        length = min(max(int(x.lens[s]), 0), x.width * x.ps)
        for i in range(n):
            row = s * n + i
            if i >= m:
                assert (got[row] == (qn[row] if in_place else 7.0)).all()
                continue
            slot = length - m + i
            pos = slot if positions is None else int(positions[row])
            for h, gain, src in ((0, gains[0], qn[row]), (1, gains[1], kn[row])):
                y = orot.norm(src, _np(gain), eps) if norms else src
                ref = orot.rotate(y, pos, freq, factor, interleaved)
                tol = _bound(y, ref, freq, pos, norms, D, x.bf16, factor)
                if h == 0:
                    assert (np.abs(got[row] - ref) <= tol).all(), (s, i, np.abs(got[row] - ref).max())
                elif slot >= 0 and 0 <= x.pages[s, slot // x.ps] < x.n_pages:
                    p, at = x.pages[s, slot // x.ps], slot % x.ps
                    assert (np.abs(pools[0][layer, p, :, at] - ref) <= tol).all(), (s, i)
                    wk[layer, p, :, at] = pools[0][layer, p, :, at]
                    wv[layer, p, :, :, at] = vn[row]
    assert np.array_equal(pools[0], wk) and np.array_equal(pools[1], wv)  # nothing else was written
    if not in_place:
        assert t.equal(rows, before)
    else:
        keep = t.ones_like(rows, dtype=t.bool)
        keep[:, :hq * D] = False
        assert t.equal(rows[keep], before[keep])
    x.pk, x.pv = pools


def _case(rgd, S, n, D=64, hk=2, ps=16, bf16=True, seed=0, most=60):
    x = Case(rgd, S, -(-(most + n) // ps) + 1, S * (-(-(most + n) // ps) + 1), hk=hk, d=D, ps=ps, bf16=bf16, seed=seed)
    new = x.r.integers(0, n + 1, S)
    new[0] = n
    assert x.reserve(np.maximum(x.r.integers(0, most, S), new))
    return x, new


@pytest.mark.parametrize("bf16", [True, False])
@pytest.mark.parametrize("D,dim", [(32, 32), (64, 64), (128, 128), (64, 32), (128, 54), (32, 2), (128, 118), (64, 0)])
@pytest.mark.parametrize("interleaved", [False, True])
def test_layouts_and_parts_of_a_head(rgd, bf16, D, dim, interleaved):
    x, new = _case(rgd, 4, 5, D=D, bf16=bf16, seed=D + dim)
    _run(rgd, x, 5, new, dim, interleaved)


@pytest.mark.parametrize("bf16,D,ps,hk,G,n,stride", [
    (True, 128, 16, 8, 4, 1, 0), (True, 64, 32, 1, 8, 3, 64), (True, 128, 48, 2, 5, 17, 8), (False, 128, 16, 3, 1, 33, 4),
    (False, 32, 64, 2, 16, 70, 0), (True, 32, 16, 1, 1, 100, 8), (True, 128, 64, 2, 2, 257, 0)])
@pytest.mark.parametrize("norms", [True, False])
def test_heads_pages_counts_and_strides(rgd, bf16, D, ps, hk, G, n, stride, norms):
    x, new = _case(rgd, 5, n, D=D, hk=hk, ps=ps, bf16=bf16, seed=n + G)
    _run(rgd, x, n, new, D, G=G, norms=norms, stride=stride)


@pytest.mark.parametrize("bf16", [True, False])
@pytest.mark.parametrize("interleaved", [False, True])
def test_in_place(rgd, bf16, interleaved):
    x, new = _case(rgd, 3, 20, D=128, bf16=bf16, seed=5)
    _run(rgd, x, 20, new, 128, interleaved, G=3, in_place=True)


@pytest.mark.parametrize("how", [("linear", 4.0), ("base", 4.0), ("by_rotations", 8.0, 8192, 1.0, 4.0),
                                 ("by_index", 16.0, 8192, 1.0, 32.0)])
@pytest.mark.parametrize("bf16", [True, False])
def test_scaled_frequencies_and_given_positions(rgd, how, bf16):
    x, new = _case(rgd, 3, 4, D=128, bf16=bf16, seed=7)
    far = np.array([0, 1, 131071, 1 << 20, -1, -4096, 7, (1 << 30) + 1, 2**31 - 1, -2**31, 12345678, 99])
    _run(rgd, x, 4, new, 128, how=how, positions=far)


def test_every_sequence_new_and_all_slots(rgd):
    x = Case(rgd, 3, 3, 9, hk=2, d=64, seed=8)
    assert x.reserve([48, 48, 48])
    _run(rgd, x, 48, None, 64)


def test_tokens_before_the_cache_and_bad_pages(rgd):
    """More new tokens than positions: the first ones have their q and nothing else; pages outside the pool are left out."""
    t = torch()
    x = Case(rgd, 3, 3, 9, hk=2, d=64, seed=9)
    assert x.reserve([20, 40, 33])
    x.pages[1, 1], x.pages[2, 0] = -1, 99
    x.c.pages.copy_(_i32(x.pages))
    x.lens = np.array([20, 40, 5000])  # clamps to 48
    x.c.lens.copy_(_i32(x.lens))
    x.pages[2, 2] = -5
    x.c.pages.copy_(_i32(x.pages))
    _run(rgd, x, 37, [37, 37, 37], 64)
    x.lens = np.array([-3, 40, 48])
    x.c.lens.copy_(_i32(x.lens))
    _run(rgd, x, 3, [3, -1, 9], 64, interleaved=True)
    t.cuda.synchronize()


@pytest.mark.parametrize("bf16", [True, False])
def test_norms_alone_of_small_and_large_rows(rgd, bf16):
    x, new = _case(rgd, 3, 6, D=128, bf16=bf16, seed=10)
    for spread in (1e-6, 1e6):
        _run(rgd, x, 6, new, 0, spread=spread)
    _run(rgd, x, 6, new, 128, spread=1e-6, eps=0.0, scale=1.25)


def test_values_that_are_not_finite_stay_in_their_row(rgd):
    t = torch()
    x, _ = _case(rgd, 2, 2, D=64, seed=11)
    q, k, v = (t.randn(4, h, 64, device="cuda").bfloat16() for h in (4, 2, 2))
    rot = rgd.Rotary(64, 1e4)
    g = t.ones(64, device="cuda")
    want = t.empty_like(q)
    rgd.paged_append_rotated(x.c, 0, q, k, v, 2, rot, want, q_norm=g, k_norm=g)
    bad, got = q.clone(), t.empty_like(q)
    bad[1, 2, 5], bad[2, 0, 60] = float("nan"), float("inf")
    rgd.paged_append_rotated(x.c, 0, bad, k, v, 2, rot, got, q_norm=g, k_norm=g)
    same = t.ones(4, 4, dtype=t.bool)
    same[1, 2] = same[2, 0] = False
    assert t.equal(got[same.cuda()], want[same.cuda()]) and t.isnan(got[1, 2]).all() and t.isnan(got[2, 0]).any()


def test_it_is_the_append_where_nothing_is_turned(rgd):
    t = torch()
    x, new = _case(rgd, 4, 9, D=128, hk=2, ps=32, seed=12)
    q, k, v = (t.randn(36, h, 128, device="cuda").bfloat16() for h in (4, 2, 2))
    rgd.paged_append(x.c, 0, k, v, 9, _i32(new))
    pk, pv = x.c.pool_k.clone(), x.c.pool_v.clone()
    x.c.pool_k[0].zero_(), x.c.pool_v[0].zero_()
    out = t.zeros_like(q)
    rgd.paged_append_rotated(x.c, 0, q, k, v, 9, None, out, n_new=_i32(new))
    row = t.from_numpy(np.arange(9)[None] < new[:, None]).view(-1).cuda()
    assert t.equal(out[row], q[row]) and (out[~row] == 0).all()
    written = x.c.pool_k[0] != 0
    assert written.any() and t.equal(x.c.pool_k[0][written], pk[0][written])
    written = x.c.pool_v[0] != 0
    assert t.equal(x.c.pool_v[0][written], pv[0][written])


def test_offsets_beyond_32_bits(rgd):
    """Rows and a layer's pools further than 2^32 bytes from their starts."""
    t = torch()
    x = Case(rgd, 2, 2, 4, layers=2, hk=1, d=128, seed=13)
    x.c = rgd.PagedCache(t.zeros(2, 1 << 20, 1, 16, 128, dtype=t.bfloat16, device="cuda"),
                         t.zeros(2, 1 << 20, 1, 128, 16, dtype=t.bfloat16, device="cuda"),
                         _i32([[(1 << 20) - 1, 0], [(1 << 20) - 3, 7]]), _i32([5, 17]), t.zeros(1 << 20, dtype=t.int32, device="cuda"), _i32([0]))
    rows = t.empty(2, 1 << 31, dtype=t.bfloat16, device="cuda")
    rows[:, :512] = t.randn(2, 512, device="cuda").bfloat16()
    qkv = rows[:, :512].unflatten(1, (4, 128))
    rot, out = rgd.Rotary(128, 1e4), t.zeros(2, 2, 128, dtype=t.bfloat16, device="cuda")
    rgd.paged_append_rotated(x.c, 1, qkv[:, :2], qkv[:, 2:3], qkv[:, 3:], 1, rot, out)
    for s, pos in ((0, 4), (1, 16)):
        page, slot = ((1 << 20) - 1, 4) if s == 0 else (7, 0)
        f, _ = orot.frequencies(128, 1e4)
        for src, got in ((qkv[s, :2], out[s]), (qkv[s, 2:3], x.c.pool_k[1, page, :, slot])):
            y = _np(src)
            ref = orot.rotate(y, pos, f)
            assert (np.abs(_np(got) - ref) <= _bound(y, ref, f, pos, False, 128, True, 1.0)).all()
        assert t.equal(x.c.pool_v[1, page, 0, :, slot], qkv[s, 3])
    assert int((x.c.pool_k != 0).sum()) <= 256 and int((x.c.pool_v != 0).sum()) <= 256


def test_binding_refuses_wrong_tensors(rgd):
    t = torch()
    x, _ = _case(rgd, 2, 3, D=64, seed=14)
    mk = lambda h, dt=t.bfloat16: t.zeros(6, h, 64, dtype=dt, device="cuda")  # noqa: E731
    good = dict(layer=0, q=mk(4), k=mk(2), v=mk(2), n=3, rotary=rgd.Rotary(64, 1e4), q_out=mk(4), n_new=_i32([1, 2]),
                positions=_i32([0] * 6), q_norm=t.ones(64, device="cuda"), k_norm=t.ones(64, device="cuda"))
    rgd.paged_append_rotated(x.c, **good)
    for kw in (dict(q=None), dict(k=None), dict(v=mk(2, t.float32)), dict(q=mk(3)), dict(k=mk(4)), dict(q_out=mk(2)), dict(n=2),
               dict(q_out=None), dict(n_new=_i32([1])), dict(n_new=t.zeros(2, device="cuda")), dict(positions=_i32([0] * 5)),
               dict(positions=_i32([0] * 6).cpu()), dict(q_norm=t.ones(32, device="cuda")), dict(k_norm=t.ones(64, device="cuda").bfloat16()),
               dict(layer=5), dict(layer=1 << 33), dict(eps=-1.0), dict(rotary=rgd.Rotary(128, 1e4)), dict(q=good["q_out"][:, :, ::2])):
        with pytest.raises(rgd.RGDError):
            rgd.paged_append_rotated(x.c, **{**good, **kw})


@pytest.mark.parametrize("bf16,D,hk,n", [(True, 32, 3, 190), (False, 128, 4, 100), (True, 64, 6, 150)])
def test_more_tokens_than_the_chip_holds(rgd, bf16, D, hk, n):
    """Enough blocks of positions that a workgroup takes several KV heads."""
    x, new = _case(rgd, 64, n, D=D, hk=hk, bf16=bf16, seed=n)
    _run(rgd, x, n, new, D, interleaved=hk == 6, in_place=hk == 4, stride=8, G=1)
