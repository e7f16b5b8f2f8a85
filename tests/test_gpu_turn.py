"""The operators of a turn together, as a decoder uses them: room for the new tokens, what the sequences share, per layer
the append with head norms and rotary positions and the attention over shared pages, and the draw under limits.  A small
decoder of random weights runs prompts, forks, steps of one token (captured once and replayed) and a ragged turn of several.
A float64 form follows it: it keeps every sequence's keys and values by themselves, without pages or groups, and checks
each operator's results from the rows that the decoder gave it, which bounds each by that operator's own roundings."""
import numpy as np
import pytest

from oracle import rotary as orot
from oracle import truncate as otr
from tests.gpu_common import torch
from tests.test_gpu_paged import Case, _dt, _i32, _np

pytestmark = pytest.mark.gpu
U = 2.0**-24  # half a step of fp32
L, HQ, HK, D, DM, V = 2, 4, 2, 32, 64, 97


@pytest.fixture(scope="module")
def rgd():
    import paper_2607_20791_amd as m
    return m


class Weights:
    def __init__(self, seed):
        r = np.random.default_rng(seed)
        f = lambda *s, by=1.0: (r.standard_normal(s) * by).astype(np.float32)  # noqa: E731
        self.emb, self.head = f(V, DM), f(DM, V, by=0.4)
        self.w = [f(DM, (HQ + 2 * HK) * D, by=DM**-0.5) for _ in range(L)]
        self.o = [f(HQ * D, DM, by=(HQ * D)**-0.5) for _ in range(L)]
        self.gain = [(1 + 0.2 * r.standard_normal((2, D))).astype(np.float32) for _ in range(L)]


class Follow:
    def __init__(self, w, S, bf16, eps):
        self.w, self.b, self.bf16, self.eps = w, 2.0**-8 if bf16 else U, bf16, eps
        self.freq, self.scale = orot.frequencies(D, 10000.0, "by_rotations", 4.0, 32.0, 1.0, 4.0)
        self.kv = [[[] for _ in range(L)] for _ in range(S)]  # per sequence and layer: (k, v) of each position

    def length(self, s):
        return len(self.kv[s][0])

    def fork(self, parent):
        self.kv = [[list(layer) for layer in self.kv[p]] for p in parent]

    def rotated(self, x, gain, pos):
        """Norm: (D / 8 + 7) u of a value, a sum of squares, its root, a division and two products; rotation: 10 u of both
        values of a pair; then half a step of the cache's type."""
        y = orot.norm(x, gain.astype(np.float64), self.eps)
        z = orot.rotate(y, pos, self.freq, self.scale)
        both = (np.abs(y) + np.abs(np.roll(y, D // 2, -1))) * self.scale
        return z, self.b * np.abs(z) + (D / 8 + 17) * U * both

    def attend(self, s, layer, q, seen):
        """Scores: (D + 2) u of the absolute sum of products, at most e; a weight changes by that, in numerator and
        denominator, by its exponent's rounding, 3 u of the score, by a rounding for each position, by 2^-16 as a pair of bf16,
        and by 8 u besides; then half a step of the cache's type."""
        k, v = (np.stack([c[i] for c in self.kv[s][layer][:seen]]) for i in (0, 1))
        out, bound = np.zeros((HQ, D)), np.zeros((HQ, D))
        for h in range(HQ):
            g = h // (HQ // HK)
            sc = k[:, g] @ q[h] / np.sqrt(D)
            e = (D + 2) * U * (np.abs(k[:, g]) @ np.abs(q[h])).max() / np.sqrt(D)
            p = np.exp(sc - sc.max())
            p /= p.sum()
            out[h] = p @ v[:, g]
            rel = 2 * e + (3 * np.abs(sc).max() + 8 + 2 * seen) * U + (2.0**-16 if self.bf16 else 0)
            bound[h] = rel * (p @ np.abs(v[:, g])) + self.b * np.abs(out[h])
        return out, bound


class Run:
    """The decoder on the GPU, over pages."""

    def __init__(self, rgd, w, x, bf16, eps, most):
        t = torch()
        self.rgd, self.x, self.eps, self.dt = rgd, x, eps, _dt(bf16)
        up = lambda a: t.from_numpy(np.ascontiguousarray(a)).cuda()  # noqa: E731
        self.emb, self.head, self.w, self.o = up(w.emb), up(w.head), [up(a) for a in w.w], [up(a) for a in w.o]
        self.gain = [up(a) for a in w.gain]
        self.rotary = rgd.Rotary(D, 10000.0, scaling=rgd.RotaryScaling("by_rotations", 4.0, 32.0, 1.0, 4.0))
        S = x.S
        self.granted = t.zeros(S, dtype=t.int32, device="cuda")
        self.shared = t.zeros(S, dtype=t.int32, device="cuda")
        self.out, self.logp = t.zeros(S, dtype=t.int32, device="cuda"), t.zeros(S, device="cuda")
        self.u, self.z = t.zeros(S, device="cuda"), t.zeros(S, V, device="cuda")
        self.T = t.tensor([0.7, 1.0, 0.0, 1.3, 0.9, 1.0], device="cuda")
        self.top_k, self.top_p = _i32([0, 20, 0, 5, 0, 90]), t.tensor([0.9, 1.0, 1.0, 0.8, 1.0, 0.95], device="cuda")
        self.min_p = t.tensor([0.0, 0.0, 0.0, 0.0, 0.05, 0.01], device="cuda")
        mem = lambda n: t.empty(n, dtype=t.uint8, device="cuda")  # noqa: E731
        self.plan = mem(max(rgd.paged_share_bytes(x.c, n, HQ) for n in most))
        self.ws = mem(max(rgd.paged_attention_shared_workspace_bytes(x.c, n, HQ) for n in most))
        self.ws_draw = mem(rgd.sample_truncated_workspace_bytes(S, V))
        self.slot = t.arange(S, device="cuda")
        rows = {n: S * n for n in most}
        # of each layer: the projection's rows, the queries as attention reads them, and its output
        self.seen = {n: [[t.zeros(m, w, dtype=self.dt, device="cuda") for w in ((HQ + 2 * HK) * D, HQ * D, HQ * D)]
                         for _ in range(L)] for n, m in rows.items()}

    def turn(self, n, tokens, grow, group):
        """tokens [S * n]: the ids of every sequence's row."""
        rgd, c, t = self.rgd, self.x.c, torch()
        rgd.paged_reserve(c, grow, self.x.ws, self.granted)
        rgd.paged_share(c, n, self.granted, HQ, group, self.plan, self.shared)
        h = self.emb.index_select(0, tokens)
        for l in range(L):
            seen = self.seen[n][l]
            qkv = (h @ self.w[l]).to(self.dt).unflatten(1, (HQ + 2 * HK, D))
            seen[0].copy_(qkv.flatten(1))
            q, k, v = qkv[:, :HQ], qkv[:, HQ:HQ + HK], qkv[:, HQ + HK:]
            rgd.paged_append_rotated(c, l, q, k, v, n, self.rotary, q, n_new=self.granted, q_norm=self.gain[l][0], k_norm=self.gain[l][1],
                                     eps=self.eps)
            seen[1].copy_(q.flatten(1))
            rgd.paged_attention_shared(c, l, q, n, self.plan, self.ws, seen[2])
            h = h + seen[2].float() @ self.o[l]
        last = self.slot * n + (self.granted - 1).clamp(min=0)
        self.z.copy_(h.index_select(0, last) @ self.head)
        rgd.sample_truncated(self.z, self.u, self.ws_draw, self.out, self.T, self.top_k, self.top_p, self.min_p, self.logp)


@pytest.mark.parametrize("bf16", [False, True])
def test_decoder_of_forked_sequences(rgd, bf16):
    t = torch()
    S, eps, r, w = 6, 1e-5, np.random.default_rng(5), Weights(7)
    x = Case(rgd, S, 5, 20, layers=L, hk=HK, d=D, bf16=bf16, seed=3)
    x.c.pool_k.fill_(float("nan")), x.c.pool_v.fill_(float("nan"))
    ref, run = Follow(w, S, bf16, eps), Run(rgd, w, x, bf16, eps, (40, 3, 1))
    group = _i32([0, 0, 0, 1, 1, 1])

    def check(n, counts):
        """After a turn in which sequence s had counts[s] new tokens."""
        t.cuda.synchronize()
        assert int(x.c.status[0]) == 0
        pages, lens, pool_k, pool_v = x.c.pages.cpu().numpy(), x.c.lens.cpu().numpy(), _np(x.c.pool_k), _np(x.c.pool_v)
        seen = [[_np(a).reshape(S, n, -1, D) for a in layer] for layer in run.seen[n]]
        for s, m in enumerate(counts):
            had = ref.length(s)
            assert lens[s] == had + m
            for l in range(L):
                rows, q, att = (a[s] for a in seen[l])
                for i in range(m):
                    pos = had + i
                    want, bound = ref.rotated(rows[i, :HQ], w.gain[l][0], pos)
                    assert (np.abs(q[i] - want) <= bound).all(), (s, l, i)
                    want, bound = ref.rotated(rows[i, HQ:HQ + HK], w.gain[l][1], pos)
                    at = pages[s, pos // x.ps], slice(None), pos % x.ps
                    k = pool_k[l][at]
                    assert (np.abs(k - want) <= bound).all(), (s, l, i)
                    ref.kv[s][l].append((k, rows[i, HQ + HK:]))
                for pos, (k, v) in enumerate(ref.kv[s][l]):  # the pages hold all of it
                    page, slot = pages[s, pos // x.ps], pos % x.ps
                    assert np.array_equal(pool_k[l, page, :, slot], k) and np.array_equal(pool_v[l, page, :, :, slot], v), (s, l, pos)
                for i in range(m):
                    want, bound = ref.attend(s, l, q[i], had + i + 1)
                    assert (np.abs(att[i] - want) <= bound).all(), (s, l, i, np.abs(att[i] - want).max(), bound.min())
        z, out, logp, u = _np(run.z), run.out.cpu().numpy(), _np(run.logp), _np(run.u)
        par = [_np(a) for a in (run.T, run.top_k, run.top_p, run.min_p)]
        for s in range(S):
            d = otr.draw(z[s], u[s], *(p[s] for p in par))
            assert d.margin > V * 2.0**-43 and out[s] == d.token, (s, out[s], d)
            assert abs(logp[s] - d.logp) <= 4 * U * max(1.0, abs(d.logp))

    def uniforms():
        run.u.copy_(t.from_numpy(r.random(S, dtype=np.float32)))

    # two prompts, in the slots that the forks start from
    prompts = [r.integers(0, V, 40), r.integers(0, V, 23)]
    counts = [40, 0, 0, 23, 0, 0]
    tokens = np.zeros((S, 40), int)
    tokens[0], tokens[3, :23] = prompts
    uniforms()
    run.turn(40, _i32(tokens.ravel()), _i32(counts), group)
    check(40, counts)
    parent = [0, 0, 0, 3, 3, 3]
    rgd.paged_select(x.c, _i32(parent), None, x.ws)
    ref.fork(parent)
    given = run.out.index_select(0, t.tensor(parent, device="cuda"))

    one = _i32([1] * S)

    def step():
        run.turn(1, given, one, group)
        given.copy_(run.out)

    uniforms()
    side = t.cuda.Stream()
    side.wait_stream(t.cuda.current_stream())
    with t.cuda.stream(side):  # once eagerly, on a stream of its own
        step()
    t.cuda.current_stream().wait_stream(side)
    check(1, [1] * S)
    assert run.shared.tolist() == [32] * 3 + [16] * 3
    graph = t.cuda.CUDAGraph()
    with t.cuda.graph(graph):
        step()
    for i in range(9):
        uniforms()
        graph.replay()
        check(1, [1] * S)
        if i == 4:  # a branch is given up for another of its prompt's
            parent = [0, 0, 2, 3, 4, 3]
            rgd.paged_select(x.c, _i32(parent), None, x.ws)
            ref.fork(parent)
            given.copy_(given.index_select(0, t.tensor(parent, device="cuda")))
    # several tokens of some sequences, then steps again
    counts = [3, 0, 1, 2, 3, 1]
    tokens = r.integers(0, V, (S, 3))
    uniforms()
    run.turn(3, _i32(tokens.ravel()), _i32(counts), group)
    check(3, counts)
    given.copy_(run.out)
    for _ in range(2):
        uniforms()
        graph.replay()
        check(1, [1] * S)
