"""Refusals of the rotated append, of the shared attention and of the sampler with per-row limits: before any HIP
call, so they run without a GPU (no pointer here is ever followed)."""
import ctypes as C

import numpy as np
import pytest

INVALID = 1


@pytest.fixture(scope="module")
def rgd():
    import paper_2607_20791_amd as m
    return m


GOOD = dict(n_layers=2, n_pages=8, n_kv_heads=2, page_size=16, head_dim=64, dtype=1, max_seqs=3, max_pages=4,
            pool_k=0x100000, pool_v=0x200000, pages=0x300000, lens=0x301000, refs=0x302000, status=0x303000)


def _at(x):
    return C.c_void_p(x)


def _desc(rgd, **kw):
    return C.byref(rgd.PagedCacheDesc(**{**GOOD, **kw}))


def _rotary(rgd, dim=64, scale=1.0, freq=None):
    f = (C.c_double * 64)(*([0.1] * 64 if freq is None else freq))
    return rgd.RotaryDesc(dim, 0, scale, f)


Q, K, V, OUT = 0x400000, 0x410000, 0x420000, 0x430000


def _append(rgd, desc=None, **kw):
    a = dict(layer=0, q=Q, k=K, v=V, ldq=256, ldk=128, ldv=128, n=2, n_new=0x500000, heads=4, positions=0x501000,
             rotary=_rotary(rgd), q_norm=0x502000, k_norm=0x503000, eps=1e-5, out=OUT, ldo=256)
    a.update(kw)
    return rgd.lib.rgd_paged_append_rotated(
        desc or _desc(rgd), a["layer"], _at(a["q"]), _at(a["k"]), _at(a["v"]), a["ldq"], a["ldk"], a["ldv"], a["n"],
        _at(a["n_new"]), a["heads"], _at(a["positions"]), a["rotary"] and C.byref(a["rotary"]), _at(a["q_norm"]),
        _at(a["k_norm"]), a["eps"], _at(a["out"]), a["ldo"], None)


def test_rotated_append_arguments(rgd):
    bad = [dict(layer=2), dict(layer=-1), dict(q=None), dict(k=None), dict(v=None), dict(out=None), dict(ldq=255), dict(ldk=127),
           dict(ldv=64), dict(ldo=128), dict(ldq=260), dict(q=Q + 8), dict(out=OUT + 8), dict(n=0), dict(n=1 << 23),
           dict(heads=0), dict(heads=3), dict(heads=2048), dict(eps=-1.0), dict(eps=float("nan")), dict(eps=float("inf")),
           dict(rotary=_rotary(rgd, 63)), dict(rotary=_rotary(rgd, 66)), dict(rotary=_rotary(rgd, -2)),
           dict(rotary=_rotary(rgd, 64, float("nan"))), dict(rotary=_rotary(rgd, 64, 1.0, [0.1] * 31 + [float("inf")] + [0] * 32)),
           dict(rotary=rgd.RotaryDesc(64, 0, 1.0, None)), dict(ldq=1 << 41)]
    for kw in bad:
        assert _append(rgd, **kw) == INVALID and rgd.lib.rgd_last_error(), kw
    assert _append(rgd, C.byref(rgd.PagedCacheDesc(**{**GOOD, "head_dim": 48}))) == INVALID
    assert rgd.lib.rgd_paged_append_rotated(None, 0, *[None] * 3, 0, 0, 0, 1, None, 1, None, None, None, None, 0.0, None, 0, None) == INVALID


def test_rotated_append_refuses_buffers_that_overlap(rgd):
    # 3 sequences of 2 rows of 4 heads of 64 in bf16: q_out has 6 * 512 bytes
    for kw in (dict(out=Q + 16), dict(out=Q, ldo=264), dict(out=K), dict(out=V - 512), dict(out=0x100000), dict(out=0x301000 - 64),
               dict(out=0x500000 - 16), dict(out=0x501000), dict(out=0x502000 - 3056), dict(out=0x503000), dict(k=0x100000),
               dict(q=0x200000), dict(v=0x300000), dict(positions=0x301000), dict(q_norm=0x302000), dict(n_new=0x301000)):
        assert _append(rgd, **kw) == INVALID and b"overlap" in rgd.lib.rgd_last_error(), kw
    # rows of a fused projection [q | k | v] of 512 + 256 + 256 bytes: q_out over k's rows, or reaching into them
    fused = dict(q=Q, k=Q + 512, v=Q + 768, ldq=512, ldk=512, ldv=512, ldo=512)
    for out in (Q + 512, Q + 256, Q - 512 - 16, Q + 1024 - 16, Q + 768):
        assert _append(rgd, **{**fused, "out": out}) == INVALID and b"overlap" in rgd.lib.rgd_last_error(), out - Q


def test_share_and_shared_attention_arguments(rgd):
    lib, d = rgd.lib, _desc(rgd)
    plan, ws, q, out, lse, group = 0x600000, 0x700000, 0x800000, 0x900000, 0xA00000, 0xB00000
    assert lib.rgd_paged_share_bytes(d, 2, 4) > 0 and lib.rgd_paged_attention_shared_workspace_bytes(d, 2, 4) > 0
    assert lib.rgd_last_error() == b""
    for n, heads in ((0, 4), (1025, 4), (2, 0), (2, 3), (2, 2048)):
        assert lib.rgd_paged_share_bytes(d, n, heads) == 0 and lib.rgd_last_error()
        assert lib.rgd_paged_attention_shared_workspace_bytes(d, n, heads) == 0
        assert lib.rgd_paged_share(d, n, None, heads, None, _at(plan), None, None) == INVALID
        assert lib.rgd_paged_attention_shared(d, 0, _at(q), 64 * max(heads, 1), n, heads, _at(plan), _at(ws), _at(out),
                                              None, None) == INVALID
    many = _desc(rgd, max_seqs=4096, max_pages=1)
    assert lib.rgd_paged_share_bytes(many, 512, 4) == 0 and lib.rgd_paged_share_bytes(many, 256, 4) > 0
    for bad in (dict(head_dim=48), dict(max_seqs=0), dict(pool_k=None)):
        assert lib.rgd_paged_share_bytes(_desc(rgd, **bad), 2, 4) == 0
    share = lambda **k: lib.rgd_paged_share(d, 2, _at(k.get("n_new")), 4, _at(k.get("group", group)), _at(k.get("plan", plan)),  # noqa: E731
                                            _at(k.get("shared")), None)
    for kw in (dict(plan=None), dict(plan=plan + 16), dict(group=plan), dict(n_new=plan + 64), dict(shared=plan),
               dict(shared=group), dict(plan=0x100000), dict(shared=0x301000)):
        assert share(**kw) == INVALID and lib.rgd_last_error(), kw
    def attend(**k):
        a = dict(layer=0, q=q, ldq=256, plan=plan, ws=ws, out=out, lse=lse)
        a.update(k)
        return lib.rgd_paged_attention_shared(d, a["layer"], _at(a["q"]), a["ldq"], 2, 4, _at(a["plan"]), _at(a["ws"]),
                                              _at(a["out"]), _at(a["lse"]), None)
    for kw in (dict(layer=2), dict(layer=-1), dict(q=None), dict(plan=None), dict(ws=None), dict(out=None), dict(ldq=128),
               dict(ldq=257), dict(q=q + 8), dict(out=out + 8), dict(ws=ws + 16), dict(plan=plan + 64), dict(out=q),
               dict(lse=out + 64), dict(ws=plan), dict(out=plan), dict(out=0x100000), dict(ws=0x300000), dict(lse=q + 16)):
        assert attend(**kw) == INVALID and lib.rgd_last_error(), kw
    assert lib.rgd_paged_share(None, 1, None, 1, None, _at(plan), None, None) == INVALID
    assert lib.rgd_paged_attention_shared(None, 0, _at(q), 64, 1, 1, _at(plan), _at(ws), _at(out), None, None) == INVALID


def test_sampler_arguments(rgd):
    lib = rgd.lib
    assert lib.rgd_sample_truncated_workspace_bytes(1, 1) > 0 and lib.rgd_sample_truncated_workspace_bytes(65536, 1 << 20) > 0
    for R, V in ((0, 8), (-1, 8), (65537, 8), (1, 0), (1, (1 << 20) + 1)):
        assert lib.rgd_sample_truncated_workspace_bytes(R, V) == 0
    z, T, k, p, m, u, ws, out, logp = (0x100000 * (i + 1) for i in range(9))

    def draw(**kw):
        a = dict(z=z, ldz=1000, R=4, V=1000, T=T, k=k, p=p, m=m, u=u, ws=ws, out=out, logp=logp)
        a.update(kw)
        return lib.rgd_sample_truncated(_at(a["z"]), a["ldz"], a["R"], a["V"], *(_at(a[n]) for n in ("T", "k", "p", "m", "u", "ws", "out", "logp")), None)

    for kw in (dict(z=None), dict(u=None), dict(ws=None), dict(out=None), dict(R=0), dict(V=0), dict(R=65537), dict(V=(1 << 20) + 1),
               dict(ldz=999), dict(ldz=1 << 41), dict(ws=ws + 16), dict(out=z + 64), dict(out=u), dict(logp=out), dict(logp=T),
               dict(ws=z), dict(out=ws), dict(out=k + 8), dict(logp=p), dict(out=m)):
        assert draw(**kw) == INVALID and lib.rgd_last_error(), kw


@pytest.mark.parametrize("V", [1, 700, 5000, 20000, 50257, 152064, 1 << 20])
def test_a_samplers_workspace_serves_fewer_rows_too(rgd, V):
    sizes = [rgd.sample_truncated_workspace_bytes(R, V) for R in list(range(1, 1100)) + [4096, 65536]]
    assert all(a <= b for a, b in zip(sizes, sizes[1:]))


def test_binding_numbers_beyond_31_bits_are_refused(rgd):
    for fn in (lambda: rgd.sample_truncated_workspace_bytes(1 << 32, 8), lambda: rgd.sample_truncated_workspace_bytes(1, 1 << 33),
               lambda: rgd.Rotary((1 << 32) + 64, 1e4)):
        with pytest.raises(rgd.RGDError):
            fn()
    assert np.isfinite(rgd.Rotary(64, 1e4).scale)
