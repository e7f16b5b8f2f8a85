"""Refusals of the paged-sequence and draft-verification entry points: before any
HIP call, so they run without a GPU (no pointer here is ever followed)."""
import ctypes as C

import pytest

INVALID = 1


@pytest.fixture(scope="module")
def rgd():
    import paper_2607_20791_amd as m
    return m


GOOD = dict(n_layers=2, n_pages=8, n_kv_heads=2, page_size=16, head_dim=64, dtype=1, max_seqs=3, max_pages=4,
            pool_k=0x1000, pool_v=0x2000, pages=0x3000, lens=0x3100, refs=0x3200, status=0x3300)
WS = C.c_void_p(0x10000)
P = C.c_void_p(0x40000)
OUT = C.c_void_p(0x80000)
W2 = C.c_void_p(0x90000)


def _desc(rgd, **kw):
    return C.byref(rgd.PagedCacheDesc(**{**GOOD, **kw}))


BAD = [dict(n_layers=0), dict(n_pages=0), dict(n_pages=(1 << 20) + 1), dict(n_kv_heads=0), dict(page_size=8),
       dict(page_size=24), dict(page_size=8192), dict(head_dim=48), dict(head_dim=256), dict(dtype=2), dict(max_seqs=0),
       dict(max_seqs=65537), dict(max_pages=0), dict(max_pages=1 << 27), dict(pool_k=None), dict(pool_v=None),
       dict(pool_k=0x1008), dict(pages=None), dict(lens=None), dict(refs=None), dict(status=None)]


@pytest.mark.parametrize("kw", BAD, ids=lambda k: "-".join(f"{a}={b}" for a, b in k.items()))
def test_bad_descriptions_are_refused_everywhere(rgd, kw):
    lib, d = rgd.lib, _desc(rgd, **kw)
    assert lib.rgd_paged_workspace_bytes(d) == 0 and lib.rgd_last_error()
    assert lib.rgd_paged_attention_workspace_bytes(d, 1, 2) == 0
    assert lib.rgd_paged_select(d, P, P, WS, None) == INVALID and lib.rgd_last_error()
    assert lib.rgd_paged_reserve(d, P, WS, None) == INVALID
    assert lib.rgd_paged_compact(d, P, WS, None) == INVALID
    assert lib.rgd_paged_append(d, 0, P, P, 128, 128, 1, None, None) == INVALID
    assert lib.rgd_paged_attention(d, 0, P, 128, 1, None, 2, WS, OUT, None, None) == INVALID


def test_null_descriptions_and_arguments(rgd):
    lib, d = rgd.lib, _desc(rgd)
    off = C.c_void_p(0x10010)
    assert lib.rgd_paged_workspace_bytes(None) == 0
    assert lib.rgd_paged_workspace_bytes(d) > 0 and lib.rgd_last_error() == b""
    for rc in (lib.rgd_paged_select(None, P, P, WS, None), lib.rgd_paged_select(d, P, None, None, None),
               lib.rgd_paged_select(d, P, None, off, None), lib.rgd_paged_reserve(d, None, WS, None),
               lib.rgd_paged_reserve(d, P, None, None), lib.rgd_paged_reserve(d, P, off, None),
               lib.rgd_paged_compact(d, None, WS, None), lib.rgd_paged_compact(d, P, off, None)):
        assert rc == INVALID and lib.rgd_last_error()


def test_append_arguments(rgd):
    lib, d = rgd.lib, _desc(rgd)

    def call(layer=0, k=P, v=P, ldk=128, ldv=128, n=1):
        return lib.rgd_paged_append(d, layer, k, v, ldk, ldv, n, None, None)

    for kw in (dict(layer=2), dict(layer=-1), dict(k=None), dict(v=None), dict(ldk=127), dict(ldv=120), dict(ldk=132),
               dict(k=C.c_void_p(0x40008)), dict(n=0), dict(n=1 << 24)):
        assert call(**kw) == INVALID, kw


def test_attention_arguments(rgd):
    lib, d = rgd.lib, _desc(rgd)
    assert lib.rgd_paged_attention_workspace_bytes(d, 1, 4) > 0
    huge = _desc(rgd, max_seqs=65536, max_pages=1 << 26, n_kv_heads=1024)
    assert lib.rgd_paged_attention_workspace_bytes(huge, 1, 1024) == 0 and b"tables" in lib.rgd_last_error()
    assert lib.rgd_paged_attention_workspace_bytes(_desc(rgd, max_seqs=65536), 257, 4) == 0
    # 4096 sequences of 2^28 positions, 8 KV heads: a run of 256 would be past 31 bits of steps
    assert lib.rgd_paged_attention_workspace_bytes(
        _desc(rgd, max_seqs=4096, max_pages=65536, page_size=4096, n_kv_heads=8), 1, 512) == 0
    for n, h in ((0, 4), (1025, 4), (1, 0), (1, 3), (1, 1026)):
        assert lib.rgd_paged_attention_workspace_bytes(d, n, h) == 0

    def call(layer=0, q=P, ldq=256, n=1, heads=4, ws=WS, out=OUT):
        return lib.rgd_paged_attention(d, layer, q, ldq, n, None, heads, ws, out, None, None)

    for kw in (dict(layer=2), dict(q=None), dict(ldq=255), dict(ldq=260), dict(q=C.c_void_p(0x40002)), dict(n=0),
               dict(heads=3), dict(ws=None), dict(ws=C.c_void_p(0x10080)), dict(out=None),
               dict(out=C.c_void_p(0x80008)), dict(out=P), dict(out=C.c_void_p(0x40000 + 512))):
        assert call(**kw) == INVALID, kw


def test_verify_arguments(rgd):
    lib = rgd.lib
    for s, k, v in ((65536, 255, 32), (65536, 64, 16385), (0, 4, 100), (65537, 4, 100), (1, 0, 100), (1, 256, 100), (1, 4, 1), (1, 4, (1 << 20) + 1)):
        assert lib.rgd_verify_workspace_bytes(s, k, v) == 0
    assert lib.rgd_verify_workspace_bytes(2, 4, 101) > 0

    def call(target=P, tokens=P, S=2, K=4, V=101, T=1.0, min_p=0.1, u=P, ws=WS, out=OUT, count=OUT):
        return lib.rgd_verify_drafts(target, None, tokens, None, S, K, V, T, min_p, u, ws, out, count, None)

    for kw in (dict(out=P), dict(count=P), dict(tokens=OUT, count=W2), dict(u=C.c_void_p(0x80000 - 36), count=W2),
               dict(u=C.c_void_p(0x80000 + 36), count=W2), dict(count=C.c_void_p(0x80000 + 36))):
        assert call(**kw) == INVALID and b"overlap" in lib.rgd_last_error(), kw
    nan = float("nan")
    for kw in (dict(target=None), dict(tokens=None), dict(u=None), dict(ws=None), dict(out=None), dict(count=None),
               dict(S=0), dict(K=0), dict(V=1), dict(T=-1.0), dict(T=nan), dict(T=float("inf")), dict(min_p=1.5),
               dict(min_p=-0.1), dict(min_p=nan), dict(ws=C.c_void_p(0x10001))):
        assert call(**kw) == INVALID and lib.rgd_last_error(), kw


@pytest.mark.parametrize("kw", [dict(dtype=0, head_dim=128, max_pages=100000), dict(head_dim=128, max_pages=100000),
                                dict(head_dim=32, max_pages=100000), dict(dtype=0), dict(max_seqs=1, max_pages=1),
                                dict(max_seqs=70, max_pages=40, n_kv_heads=1)])
@pytest.mark.parametrize("group", [1, 3, 8, 20])
def test_an_attention_workspace_serves_fewer_tokens_too(rgd, kw, group):
    """The bytes for up to n tokens are enough for every smaller count."""
    kw = {"max_seqs": 64, **kw}
    d, heads = _desc(rgd, **kw), group * kw.get("n_kv_heads", GOOD["n_kv_heads"])
    need = [rgd.lib.rgd_paged_attention_workspace_bytes(d, n, heads) for n in range(1, 130)]
    assert need[0] > 0 and need == sorted(need)


def test_reserve_with_granted_arguments(rgd):
    lib, d = rgd.lib, _desc(rgd)

    def call(cache=d, grow=P, granted=OUT, ws=WS):
        return lib.rgd_paged_reserve_granted(cache, grow, granted, ws, None)

    for kw in (dict(cache=None), dict(cache=_desc(rgd, n_pages=0)), dict(grow=None), dict(granted=None), dict(ws=None),
               dict(ws=C.c_void_p(0x10010)), dict(granted=C.c_void_p(0x40000 + 8)), dict(granted=C.c_void_p(0x40000 - 8))):
        assert call(**kw) == INVALID and lib.rgd_last_error(), kw


# buffers of a cache far apart from each other and from WS, P, OUT and W2
APART = dict(pool_k=0x10000000, pool_v=0x20000000, pages=0x30000000, lens=0x31000000, refs=0x32000000, status=0x33000000)


def _at(x):
    return C.c_void_p(x)


def test_attention_refuses_buffers_that_overlap(rgd):
    lib, d = rgd.lib, _desc(rgd, **APART)
    counts = _at(0x60000)

    def call(q=P, out=OUT, ws=_at(0x1000000), lse=W2, ldq=256):
        return lib.rgd_paged_attention(d, 0, q, ldq, 2, counts, 4, ws, out, lse, None)

    need = lib.rgd_paged_attention_workspace_bytes(d, 2, 4)  # q: 6 rows of 512 bytes; lse: 96 bytes
    cases = [dict(lse=OUT), dict(lse=_at(0x80000 + 6 * 512 - 4)), dict(lse=P), dict(lse=_at(0x40000 + 6 * 512 - 4)), dict(lse=counts),
             dict(lse=_at(0x60000 - 92)), dict(out=counts), dict(ws=OUT), dict(ws=P), dict(ws=_at(0x80000 - need + 256)),
             dict(ws=W2), dict(ldq=1 << 39, out=_at(0x40000 + (1 << 40)))]
    cases += [{k: _at(a)} for k in ("out", "lse", "ws") for a in APART.values()]
    cases += [dict(out=_at(0x10000000 + 65536 - 16)), dict(lse=_at(0x10000000 - 92)), dict(ws=_at(0x32000000 - 256))]
    for kw in cases:
        assert call(**kw) == INVALID and b"overlap" in lib.rgd_last_error(), kw


def test_page_operators_refuse_buffers_that_overlap(rgd):
    lib, d = rgd.lib, _desc(rgd, **APART)
    for at in APART.values():
        for rc in (lib.rgd_paged_select(d, P, None, _at(at), None), lib.rgd_paged_reserve(d, P, _at(at), None),
                   lib.rgd_paged_reserve_granted(d, P, _at(at), WS, None), lib.rgd_paged_compact(d, OUT, _at(at), None),
                   lib.rgd_paged_compact(d, _at(at), WS, None)):
            assert rc == INVALID and b"overlap" in lib.rgd_last_error(), hex(at)
    for rc in (lib.rgd_paged_select(d, P, None, P, None), lib.rgd_paged_select(d, W2, P, P, None),
               lib.rgd_paged_reserve(d, P, P, None), lib.rgd_paged_reserve(d, _at(0x10000 + 4), WS, None),
               lib.rgd_paged_reserve_granted(d, P, WS, WS, None), lib.rgd_paged_compact(d, WS, WS, None)):
        assert rc == INVALID and b"overlap" in lib.rgd_last_error()


def test_verify_refuses_a_workspace_that_overlaps(rgd):
    lib = rgd.lib
    need = lib.rgd_verify_workspace_bytes(2, 4, 101)
    a = dict(target=0x1000000, draft=0x2000000, tokens=0x3000000, nd=0x3100000, u=0x3200000, out=0x3300000, count=0x3400000)
    for at in list(a.values()) + [a["u"] - need + 256, a["target"] + 4096 - 256]:
        p = {k: _at(v) for k, v in a.items()}
        rc = lib.rgd_verify_drafts(p["target"], p["draft"], p["tokens"], p["nd"], 2, 4, 101, 1.0, 0.1, p["u"], _at(at // 256 * 256),
                                   p["out"], p["count"], None)
        assert rc == INVALID and b"overlap" in lib.rgd_last_error(), hex(at)


def test_verify_sizes_beyond_31_bits_are_refused(rgd):
    for args in (((1 << 32) + 2, 4, 101), (2, (1 << 32) + 4, 101), (2, 4, (1 << 32) + 101)):
        with pytest.raises(rgd.RGDError):
            rgd.verify_workspace_bytes(*args)
    assert rgd.verify_workspace_bytes(2, 4, 101) > 0
