"""The sampler with per-row limits on the GPU against the float64 oracle."""
import numpy as np
import pytest

from oracle import truncate as ot
from tests.gpu_common import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def rgd():
    import paper_2607_20791_amd as m
    return m


def _gpu(a, dt=np.float32):
    return None if a is None else torch().from_numpy(np.ascontiguousarray(a, dtype=dt)).cuda()


def _run(rgd, z, u, T=None, k=None, p=None, m=None, pad=0):
    t = torch()
    R, V = z.shape
    zt = t.full((R, V + pad), 1e30, device="cuda")
    zt[:, :V] = _gpu(z)
    ws = t.empty(rgd.sample_truncated_workspace_bytes(R, V), dtype=t.uint8, device="cuda").fill_(255)
    out, logp = t.full((R,), -7, dtype=t.int32, device="cuda"), t.full((R,), 7.0, device="cuda")
    rgd.sample_truncated(zt[:, :V], _gpu(u), ws, out, T=_gpu(T), top_k=_gpu(k, np.int32), top_p=_gpu(p), min_p=_gpu(m), logp=logp)
    t.cuda.synchronize()
    return out.cpu().numpy(), logp.cpu().numpy()


def _compare(rgd, z, u, T=None, k=None, p=None, m=None, pad=0, near=0):
    """Every row's id is the oracle's, unless u or top_p meets a border of two ids by what the weights' rounding to 2^-44
    and 40 roundings of fp64 sums can move it; at most `near` rows may.  logp: a rounding of fp32, and the weights'."""
    z = np.asarray(z, np.float32)
    u = np.asarray(u, np.float32)
    out, logp = _run(rgd, z, u, T, k, p, m, pad)
    met = 0
    for r in range(len(z)):
        at = lambda a, off: off if a is None else float(np.float32(a[r]))  # noqa: E731
        d = ot.draw(z[r], u[r], at(T, 1.0), int(at(k, 0)), at(p, 1.0), at(m, 0.0))
        w = len(z[r]) * 2.0**-43 + 40 * 2.0**-53 * max(len(d.kept), 1)
        if d.margin <= w:
            met += 1
            continue
        assert out[r] == d.token, (r, out[r], d.token, d.margin)
        if np.isneginf(d.logp):
            assert np.isneginf(logp[r])
        else:
            assert abs(logp[r] - d.logp) <= 2.0**-23 * max(abs(d.logp), 1.0) + 2 * w, (r, logp[r], d.logp)
    assert met <= near
    return out


def _rows(seed, R, V, scale=2.0, likely=20):
    r = np.random.default_rng(seed)
    z = (r.standard_normal((R, V)) * scale).astype(np.float32)
    for row in z:
        row[r.integers(0, V, likely)] += (r.random(likely) * 8).astype(np.float32)
    return z, r.random(R, dtype=np.float32), r


VS = [1, 2, 3, 5, 63, 64, 65, 127, 255, 256, 257, 1000, 2047, 2048, 2049, 4097, 8191, 20011, 50257]


@pytest.mark.parametrize("V", VS)
@pytest.mark.parametrize("what", ["none", "k", "p", "m", "all"])
def test_against_the_oracle(rgd, V, what):
    z, u, r = _rows(V, 6, V)
    on = lambda name, a: a if what in (name, "all") else None  # noqa: E731
    _compare(rgd, z, u, T=[1.0, 0.5, 2.0, 3.0, 0.1, 1.0], k=on("k", [1, 2, 40, max(V // 2, 1), V, V + 5]),
             p=on("p", [0.9, 0.5, 0.99, 0.1, 0.95, 0.0]), m=on("m", [0.1, 0.02, 0.5, 0.0, 1.0, 0.3]), pad=V % 3)


@pytest.mark.parametrize("V", [131072, 151936, 262145, 1 << 20])
def test_large_vocabularies(rgd, V):
    z, u, _ = _rows(V, 4, V)
    _compare(rgd, z, u, T=[0.7, 1.0, 2.0, 4.0], k=[50, 0, 0, 100000], p=[0.95, 0.9, 0.9, 0.8], m=[0.0, 0.0, 0.0, 0.01])


@pytest.mark.parametrize("R", [1, 2, 7, 64, 200, 300])
def test_rows_with_limits_of_their_own(rgd, R):
    z, u, r = _rows(R, R, 5003)
    z[r.random(z.shape) < 0.2] = -np.inf
    pick = lambda *a: r.choice(a, R)  # noqa: E731
    _compare(rgd, z, u, T=pick(0.0, 0.3, 1.0, 2.5, -1.0), k=pick(0, -3, 1, 10, 500, 6000), p=pick(1.0, 0.5, 0.9, 2.0, 0.0),
             m=pick(0.0, 0.05, -1.0, 2.0))


def test_the_same_row_gives_the_same_id_in_any_batch(rgd):
    z, u, _ = _rows(1, 300, 30011)
    args = dict(T=np.full(300, 1.7), k=np.full(300, 3000), p=np.full(300, 0.93), m=np.full(300, 1e-4))
    whole, logp = _run(rgd, z, u, **args)
    for rows in (slice(0, 1), slice(5, 9), slice(100, 180)):
        out, lp = _run(rgd, z[rows], u[rows], **{n: a[rows] for n, a in args.items()})
        assert np.array_equal(out, whole[rows]) and np.array_equal(lp, logp[rows])


@pytest.mark.parametrize("V", [7, 300, 20000, 152064])
def test_equal_logits_go_by_their_ids(rgd, V):
    u = np.array([0.0, 0.3, 0.9999, 0.5, 0.5, 0.999], np.float32)
    z = np.zeros((6, V), np.float32)
    z[4] = -0.0
    z[5, ::2] = -0.0  # equal to 0
    # a flat row of k ids: the draw is floor(u k) where that is no border
    k = np.array([5, 7, 3, V, 0, 5])
    out = _compare(rgd, z, u, k=k, near=3)
    assert out[0] == 0 and out[2] == 2
    _compare(rgd, z, u, p=[0.31, 0.52, 0.17, 0.999, 0.0, 0.5], near=3)
    z[:, V // 2] = 1.0
    _compare(rgd, z, u, k=np.array([1, 2, 3, 4, 5, 6]), p=[0.9, 0.8, 0.7, 0.6, 0.5, 0.4], near=3)


@pytest.mark.parametrize("V", [3000, 128256])
def test_logits_of_few_values(rgd, V):
    """Rounded logits: hundreds of ids share each value, at every limit's border too."""
    z, u, r = _rows(5, 8, V)
    z = np.round(z * 2) / 2
    _compare(rgd, z, u, k=[3, 100, 1000, 0, 0, 17, 2500, 0], p=[1.0, 0.9, 0.5, 0.9, 0.3, 0.99, 0.7, 0.05], near=2)


def test_distributions_at_the_ends(rgd):
    V = 4099
    z, u, r = _rows(9, 9, V)
    z[0] = -np.inf
    z[1, 7] = np.inf
    z[2] = np.nan
    z[3] = -np.inf
    z[3, 4000] = -3.0e38      # one id left
    z[4, :] = 3.0e38          # equal ones at the top
    z[5] = np.where(np.arange(V) % 2, -np.inf, z[5])
    z[5, 1::4] = np.nan
    z[6] *= 1e30              # one has everything
    z[7] *= 1e-30             # flat but for the order
    z[8, 10:] = -np.inf
    for k in (None, np.full(9, 5), np.full(9, 100)):
        for p in (None, np.full(9, 0.9)):
            out = _compare(rgd, z, u, k=k, p=p, m=np.full(9, 1e-6), near=2)
            assert list(out[:3]) == [-1, -1, -1] and out[3] == 4000
    assert list(_run(rgd, z, u, T=np.zeros(9))[0][:3]) == [-1, -1, -1]


def test_temperatures_uniforms_and_limits_outside_their_ranges(rgd):
    z, u, r = _rows(11, 12, 1777)
    T = np.array([1e-30, 1e-45, 1e30, 3e38, np.inf, np.nan, -0.0, -np.inf, 1.0, 1.0, 1.0, 1.0], np.float32)
    u[8:] = [1.0, -0.5, np.nan, np.inf]
    ref = np.where(np.isnan(u), 0.0, np.clip(u, 0.0, 1.0 - 2.0**-24)).astype(np.float32)
    out, _ = _run(rgd, z, u, T=T)
    for i in range(12):
        if i in (2, 3, 4):  # weights that are all 1 but for less than fp64 has: u's place among the ids
            assert abs(int(out[i]) - int(float(u[i]) * 1777)) <= 1
        else:
            assert out[i] == ot.draw(z[i], ref[i], float(T[i])).token, i
    nan = np.full(12, np.nan)
    _compare(rgd, z, ref, p=nan, m=nan, k=np.full(12, -2**31))
    _compare(rgd, z, ref, p=np.full(12, -1.0), k=np.full(12, 2**31 - 1))
    _compare(rgd, z, ref, p=np.full(12, 1e-38), m=np.full(12, np.inf))


def test_rows_beyond_32_bits(rgd):
    t = torch()
    V, R = 1 << 20, 1100  # 4.6 GB
    z = t.zeros(R, V, device="cuda")
    z[:, 12345] = 30.0
    z[R - 1, 12345], z[R - 1, V - 1] = 0.0, 30.0
    ws = t.empty(rgd.sample_truncated_workspace_bytes(R, V), dtype=t.uint8, device="cuda")
    out = t.empty(R, dtype=t.int32, device="cuda")
    rgd.sample_truncated(z, t.full((R,), 0.5, device="cuda"), ws, out, top_p=t.full((R,), 0.9, device="cuda"))
    assert (out[:-1] == 12345).all() and int(out[-1]) == V - 1


def test_borders_are_exact(rgd):
    """Weights that are powers of two: sums are exact, and a u on a border goes to the next id."""
    z = np.log(np.array([[8.0, 4.0, 2.0, 1.0, 1.0]], np.float64)).astype(np.float32)
    z = np.repeat(np.array([[0.0, -1.0, -2.0, -3.0, -3.0]], np.float32), 5, 0)
    T = np.full(5, np.float32(1.0 / np.log(2.0)))  # weights 2^z but for T's rounding
    out, logp = _run(rgd, z, np.array([0.0, 0.49, 0.51, 0.76, 0.95], np.float32), T=T)
    assert list(out) == [0, 0, 1, 2, 4] and np.allclose(logp, np.log([0.5, 0.5, 0.25, 0.125, 0.0625]), atol=1e-6)
    flat = np.zeros((4, 4), np.float32)
    assert list(_run(rgd, flat, np.array([0.0, 0.25, 0.5, 0.75], np.float32))[0]) == [0, 1, 2, 3]
    assert list(_run(rgd, flat, np.array([0.75] * 4, np.float32), p=[0.25, 0.5, 0.75, 0.76])[0]) == [0, 1, 2, 3]


@pytest.mark.parametrize("T,min_p", [(1.0, 0.1), (2.0, 0.05), (0.7, 0.0)])
def test_it_is_the_verifications_draw(rgd, T, min_p):
    """Without top-k and top-p the draw is what verify_drafts draws after its drafts."""
    t = torch()
    z, u, _ = _rows(21, 16, 30000)
    target = _gpu(np.repeat(z[:, None], 2, 1))
    S, V = z.shape
    ws = t.empty(rgd.verify_workspace_bytes(S, 1, V), dtype=t.uint8, device="cuda")
    out, count = t.empty(S, 2, dtype=t.int32, device="cuda"), t.empty(S, dtype=t.int32, device="cuda")
    uu = np.stack([u, u], 1)
    rgd.verify_drafts(target, None, t.zeros(S, 1, dtype=t.int32, device="cuda"), t.zeros(S, dtype=t.int32, device="cuda"), T, min_p,
                      _gpu(uu), ws, out, count)
    got, _ = _run(rgd, z, u, T=np.full(S, T), m=np.full(S, min_p))
    assert np.array_equal(got, out[:, 0].cpu().numpy())


def test_another_stream_and_a_captured_call(rgd):
    t = torch()
    z, u, _ = _rows(31, 40, 50000)
    args = dict(T=_gpu(np.full(40, 1.5)), top_k=_gpu(np.full(40, 700), np.int32), top_p=_gpu(np.full(40, 0.9)), min_p=_gpu(np.full(40, 1e-3)))
    zt, ut = _gpu(z), _gpu(u)
    ws = t.empty(rgd.sample_truncated_workspace_bytes(40, 50000), dtype=t.uint8, device="cuda")
    mk = lambda: (t.empty(40, dtype=t.int32, device="cuda"), t.empty(40, device="cuda"))  # noqa: E731
    a, la = mk()
    rgd.sample_truncated(zt, ut, ws, a, logp=la, **args)
    t.cuda.synchronize()
    b, lb = mk()
    side = t.cuda.Stream()
    with t.cuda.stream(side):
        rgd.sample_truncated(zt, ut, ws, b, logp=lb, **args)
    side.synchronize()
    assert t.equal(a, b) and t.equal(la, lb)
    c, lc = mk()
    graph = t.cuda.CUDAGraph()
    with t.cuda.graph(graph):
        rgd.sample_truncated(zt, ut, ws, c, logp=lc, **args)
    for i in range(4):
        c.fill_(-9)
        fresh = t.roll(zt, 13 * i, 1)
        eager, le = mk()
        rgd.sample_truncated(fresh, ut, t.empty_like(ws), eager, logp=le, **args)
        old = zt.clone()
        zt.copy_(fresh)
        graph.replay()
        t.cuda.synchronize()
        assert t.equal(c, eager) and t.equal(lc, le)
        zt.copy_(old)


def test_binding_refuses_wrong_tensors(rgd):
    t = torch()
    z, u = t.zeros(3, 100, device="cuda"), t.zeros(3, device="cuda")
    ws = t.empty(rgd.sample_truncated_workspace_bytes(3, 100), dtype=t.uint8, device="cuda")
    out = t.empty(3, dtype=t.int32, device="cuda")
    rgd.sample_truncated(z, u, ws, out)
    good = dict(z=z, u=u, workspace=ws, out=out)
    for kw in (dict(z=None), dict(z=z.half()), dict(z=z.cpu()), dict(z=z[0]), dict(z=z.T.contiguous().T), dict(z=z[:, ::2]),
               dict(u=None), dict(u=u[:2]), dict(u=u.double()), dict(workspace=None), dict(workspace=ws[:8]), dict(out=out.long()),
               dict(out=None), dict(T=t.ones(2, device="cuda")), dict(top_k=u), dict(top_p=out), dict(min_p=u.cpu()),
               dict(logp=out), dict(logp=u), dict(z=z[:1].expand(3, 100))):
        with pytest.raises(rgd.RGDError):
            rgd.sample_truncated(**{**good, **kw})


@pytest.mark.parametrize("R,V", [(1024, 300), (1025, 300), (2500, 77)])
def test_more_rows_than_are_taken_at_a_time(rgd, R, V):
    z, u, r = _rows(R, R, V)
    pick = lambda *a: r.choice(a, R)  # noqa: E731
    _compare(rgd, z, u, T=pick(0.0, 0.5, 1.0), k=pick(0, 1, 10, 60), p=pick(1.0, 0.5, 0.9), m=pick(0.0, 0.05))


def test_two_captured_calls_share_a_workspace(rgd):
    """Graphs of different sizes over one workspace, replayed in turn with eager calls between."""
    t = torch()
    calls = []
    for R, V in ((3, 5000), (70, 900)):
        z, u, r = _rows(R, R, V)
        calls.append((_gpu(z), _gpu(u), t.empty(R, dtype=t.int32, device="cuda"), _gpu(r.choice([0.5, 0.9], R))))
    ws = t.empty(max(rgd.sample_truncated_workspace_bytes(*c[0].shape) for c in calls), dtype=t.uint8, device="cuda")
    want, graphs = [], []
    for z, u, out, p in calls:
        rgd.sample_truncated(z, u, ws, out, top_p=p)
        t.cuda.synchronize()
        want.append(out.clone())
        graph = t.cuda.CUDAGraph()
        with t.cuda.graph(graph):
            rgd.sample_truncated(z, u, ws, out, top_p=p)
        graphs.append(graph)
    for i in (0, 1, 1, 0, 1, 0):
        for c in calls:
            c[2].fill_(-9)
        ws.fill_(255)
        graphs[i].replay()
        t.cuda.synchronize()
        assert t.equal(calls[i][2], want[i])
        assert (calls[1 - i][2] == -9).all()


@pytest.mark.parametrize("V", [300, 30000])
def test_banned_ids_at_temperatures_near_the_largest(rgd, V):
    """T of 2^124 and more, where the range of logits that weigh anything ends below what fp32 holds: -inf weighs nothing."""
    r = np.random.default_rng(V)
    T = np.array([2e37, 5e37, 1e38, 2e37, 5e37, 1e38])
    z = r.standard_normal((6, V)) * T[:, None] / 2
    z = np.where(r.random(z.shape) < 0.7, -np.inf, np.clip(z, -3e38, 3e38)).astype(np.float32)
    least = np.exp((0.1 * T - z.max(1)) / T)  # min_p's border, a little above 0 and below top_p's
    for u in (r.random(6), np.full(6, 0.995)):
        for m in (None, least, np.array([0.2, 0.5, 0.3, 0.05, 0.6, 0.9])):
            _compare(rgd, z, u, T=T, p=np.full(6, 0.2), m=m)
            _compare(rgd, z, u, T=T, k=[3, V // 5, V // 4, 40, 7, 1], m=m)
            _compare(rgd, z, u, T=T, k=[30, V // 5, V // 4, 40, 70, 10], p=[0.5, 0.6, 0.7, 0.8, 0.9, 0.3], m=m)


def _min_p_above_top_p(seed):
    """Rows of a few logits that many ids share: min_p keeps the highest of them, whose weight is within 1.5 per cent of
    what top_p keeps, on either side.  (z, u, T, top_p, min_p)"""
    r = np.random.default_rng(seed)
    z, T, p, m = np.full((16, 18000), -np.inf, np.float32), np.empty(16), np.empty(16), np.empty(16)
    for i in range(16):
        T[i] = r.choice([0.5, 0.8, 1.0, 1.3])
        values = r.integers(200, 400) / 8 - np.cumsum(np.concatenate([[0], r.integers(1, 5, 4)])) / 8
        row = np.concatenate([np.full(r.integers(1000, 3000), v) for v in values] + [values[0] - 20 - 20 * r.random(2000)])
        z[i, r.permutation(z.shape[1])[:len(row)]] = row
        cut = r.integers(1, 4)  # values that min_p keeps
        m[i] = np.exp(((values[cut - 1] + values[cut]) / 2 - values[0]) / T[i])
        w = np.exp((z[i].astype(np.float64) - values[0]) / T[i])
        p[i] = w[z[i] >= values[cut - 1]].sum() / w.sum() * (1 + r.uniform(-0.015, 0.015))
    return z, r.choice([0.9999, 0.99999, 0.998, 0.5, 0.3], 16), T, p, m


def test_min_p_above_an_estimate_of_top_ps_border(rgd):
    """6000 ids of 33.125 behind 3000 of 33.375, of which top_p keeps 2988, and min_p all."""
    r = np.random.default_rng(1)
    z = r.permutation(np.concatenate([np.full(3000, 33.375), np.full(6000, 33.125), -7 + r.random(4000)]))[None].repeat(3, 0)
    one = np.ones(3)
    # u = 0.5 of 2988 equal weights is 1494 of them: on a border
    out = _compare(rgd, z, [0.9999, 0.5, 0.997], T=0.8 * one, p=0.40427926 * one, m=0.85534531 * one, near=1)
    assert out[0] == 12943  # u behind the twelve ids that top_p drops
    for seed in range(6):
        z, u, T, p, m = _min_p_above_top_p(seed)
        # where an even number of equal logits is kept, n / 2 weights are u = 0.5 of n: on a border, in up to three of these rows
        _compare(rgd, z, u, T=T, p=p, m=m, near=3)
        _compare(rgd, z, u, T=T, k=r.choice([500, 3000, 9000, 13000], 16), p=p, m=m, near=3)



@pytest.mark.parametrize("T", [1.0, 0.7, 2.5])
def test_borders_as_near_as_the_weights_are_exact(rgd, T):
    """Two ids, and every u or top_p among four million rows that lies nearer to their border than 6e-13 of the larger one's weight,
    but not so near as the weights' rounding to 2^-44 (with their own error of 2^-46) can move it."""
    T32 = np.float32(T)
    low = -(np.arange(1 << 22, dtype=np.float32) + 1) * np.float32(2.0**-22) * T32  # weights from 1 down to 1 / e
    w = np.exp(low.astype(np.float64) / float(T32))
    for what in ("u", "p"):
        border = w / (1 + w) if what == "u" else 1 / (1 + w)
        x = border.astype(np.float32)
        off = np.abs(border - x.astype(np.float64)) * (1 + w)
        at = np.flatnonzero((off < 6e-13) & (off > 2.5e-13))
        assert len(at) >= 20
        z = np.stack([low[at], np.zeros(len(at), np.float32)], 1)
        on = np.full(len(at), T)
        if what == "u":
            _compare(rgd, z, x[at], T=on)
        else:
            _compare(rgd, z, np.zeros(len(at)), T=on, p=x[at])  # the lower id only if top_p keeps it
