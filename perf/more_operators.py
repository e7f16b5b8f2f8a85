"""Measured cases of what a turn of a paged decoder needs besides its cache's own operators: the attention of sequences
that share leading pages, the append with head norms and rotary positions, and sampling with per-row truncation.

Each case is a plain dict; `prepare` builds what a serving program holds before the call, `run` makes one pass, either in
plain torch operations or (with `own`) through the entry points of `paper_2607_20791_amd`, and `exact` computes the same
outputs in 64 bits.

Kinds:
  shared   one turn's plan of which leading pages the branches of each prompt share, then causal attention of the new
           tokens over the shared pages and the branches' own, in every layer
  rotate   the new tokens' rows of a fused projection: norms of the query and key heads, rotary positions, K and V put
           into the pages, the queries for the attention, one layer
  sample   one token per row from logits under temperature, top-k, top-p and min-p, by given uniform numbers

Lengths are spread over their range by the case alone (the seed orders them), so that a case's work is known.
"""
import math

import numpy as np
import torch

own = False


def listed():
    return [
        # two branches of a short prompt in the small fp32 decoder: launches and latency
        {"name": "shared-f32-1x2-p100", "kind": "shared", "prompts": 1, "branches": 2, "prompt_len": 100, "tail": 9, "n": 1,
         "layers": 1, "heads": 4, "kv_heads": 2, "head_dim": 64, "dtype": "f32", "page": 16},
        # 64 branches of one long prompt, one layer (the wide one-layer decoder)
        {"name": "shared-1x64-p8192", "kind": "shared", "prompts": 1, "branches": 64, "prompt_len": 8192, "tail": 128,
         "n": 1, "layers": 1, "heads": 32, "kv_heads": 8, "head_dim": 128, "dtype": "bf16", "page": 16},
        # 32 prompts with 8 branches each, four layers of a turn
        {"name": "shared-32x8-p1024", "kind": "shared", "prompts": 32, "branches": 8, "prompt_len": 1024, "tail": 256,
         "n": 1, "layers": 4, "heads": 32, "kv_heads": 8, "head_dim": 128, "dtype": "bf16", "page": 16},
        # up to four drafts and the token before them on the branches of four prompts of odd lengths, larger pages
        {"name": "shared-4x16x5-p4095", "kind": "shared", "prompts": 4, "branches": 16, "prompt_len": 4095, "tail": 100,
         "n": 5, "layers": 2, "heads": 32, "kv_heads": 8, "head_dim": 128, "dtype": "bf16", "page": 64},
        # one token of one request: the host call and a launch
        {"name": "rotate-1x1", "kind": "rotate", "seqs": 1, "n": 1, "max_len": 500, "heads": 32, "kv_heads": 8,
         "head_dim": 128, "dtype": "bf16", "page": 16, "dims": 128, "layout": "half", "norms": True, "scaling": "none",
         "ahead": 0},
        # one token of each of 64 branches, positions far beyond the trained context
        {"name": "rotate-64x1-scaled", "kind": "rotate", "seqs": 64, "n": 1, "max_len": 2048, "heads": 32, "kv_heads": 8,
         "head_dim": 128, "dtype": "bf16", "page": 16, "dims": 128, "layout": "half", "norms": True,
         "scaling": "by_index", "ahead": 1 << 20},
        # eight prompts in pieces of up to 1000 tokens
        {"name": "rotate-8x1000", "kind": "rotate", "seqs": 8, "n": 1000, "max_len": 4096, "heads": 32, "kv_heads": 8,
         "head_dim": 128, "dtype": "bf16", "page": 16, "dims": 128, "layout": "half", "norms": True,
         "scaling": "by_rotations", "ahead": 0},
        # the small fp32 decoder's heads: half of each is rotated, in pairs of neighbours
        {"name": "rotate-f32-5x333-pairs", "kind": "rotate", "seqs": 5, "n": 333, "max_len": 999, "heads": 4,
         "kv_heads": 2, "head_dim": 64, "dtype": "f32", "page": 32, "dims": 32, "layout": "interleaved", "norms": False,
         "scaling": "none", "ahead": 0},
        # one request with the usual settings of a chat
        {"name": "sample-1x128256-k50", "kind": "sample", "rows": 1, "vocab": 128256, "T": 0.7, "top_k": 50, "top_p": 0.95,
         "min_p": 0.0, "mix": False, "banned": False},
        # a batch of requests that each have settings of their own, greedy ones and banned ids among them
        {"name": "sample-64x128256-mix", "kind": "sample", "rows": 64, "vocab": 128256, "T": 1.0, "top_k": 200,
         "top_p": 0.9, "min_p": 0.05, "mix": True, "banned": True},
        # the nucleus at a high temperature over the largest vocabulary: tens of thousands of ids are kept
        {"name": "sample-256x152064-p90", "kind": "sample", "rows": 256, "vocab": 152064, "T": 2.0, "top_k": 0,
         "top_p": 0.9, "min_p": 0.0, "mix": False, "banned": False},
        # an odd vocabulary and a large k
        {"name": "sample-33x50257-k1000", "kind": "sample", "rows": 33, "vocab": 50257, "T": 1.5, "top_k": 1000,
         "top_p": 1.0, "min_p": 0.0, "mix": False, "banned": False},
    ]


def _log(rng, lo, hi):
    """An integer spread over the logarithm of [lo, hi]."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["shared", "shared", "rotate", "sample"])
    dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
    page = rng.choice([16, 16, 32, 64])
    dim = rng.choice([64, 128] if dtype == "bf16" else [32, 64, 128])
    hk = rng.choice([1, 2, 4, 8])
    hq = hk * rng.choice([1, 2, 4, 8])
    if kind == "shared":
        prompts = _log(rng, 1, 32)
        branches = _log(rng, 1, 256 // prompts)
        layers = rng.choice([1, 1, 2, 4])
        tail = _log(rng, 1, 256)
        n = rng.choice([1, 1, 1, min(rng.randint(2, 8), tail)])
        # at most what the plain form of 64 branches of 8192 positions takes
        most = 64 * 8192 * 8 * 128 // (prompts * branches * layers * hk * dim * (1 if dtype == "bf16" else 2))
        return {"kind": kind, "prompts": prompts, "branches": branches, "prompt_len": _log(rng, 1, min(8192, max(16, most - tail))),
                "tail": tail, "n": n, "layers": layers, "heads": min(hq, 32), "kv_heads": hk, "head_dim": dim,
                "dtype": dtype, "page": page}
    if kind == "rotate":
        seqs = _log(rng, 1, 64)
        n = rng.choice([1, rng.randint(2, 8), _log(rng, 9, 8000 // seqs)])
        return {"kind": kind, "seqs": seqs, "n": n, "max_len": _log(rng, max(n, 16), 4096), "heads": hq, "kv_heads": hk,
                "head_dim": dim, "dtype": dtype, "page": page, "dims": rng.choice([dim, dim, dim // 2, dim - 10]),
                "layout": rng.choice(["half", "half", "interleaved"]), "norms": rng.random() < 0.6,
                "scaling": rng.choice(["none", "linear", "base", "by_rotations", "by_index"]),
                "ahead": rng.choice([0, 0, 0, 1 << 20])}
    return {"kind": kind, "rows": _log(rng, 1, 256), "vocab": _log(rng, 8000, 152064),
            "T": rng.choice([0.0, 0.3, 0.7, 1.0, 1.5, 2.0, 3.0]), "top_k": rng.choice([0, 0, 1, 20, 50, _log(rng, 2, 5000)]),
            "top_p": rng.choice([1.0, 0.5, 0.9, 0.95, 0.99]), "min_p": rng.choice([0.0, 0.0, 0.02, 0.1]),
            "mix": rng.random() < 0.4, "banned": rng.random() < 0.3}


# ------------------------------------------------------------------- inputs --
def _dtype(c):
    return torch.bfloat16 if c["dtype"] == "bf16" else torch.float32


def _size(c):
    return 2 if c["dtype"] == "bf16" else 4


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(int(seed) * 6271 + 29)


def _normal(g, shape, std, dtype):
    """N(0, std^2) of the given type (drawn in parts: large pools need no fp32 copy)."""
    out = torch.empty(shape, dtype=dtype, device="cuda")
    flat = out.view(-1)
    for i in range(0, flat.numel(), 1 << 27):
        part = flat[i:i + (1 << 27)]
        part.copy_(torch.randn(part.numel(), generator=g, device="cuda").mul_(std))
    return out


def _spread(n, lo, hi):
    """n integers from lo to hi, spread over their logarithm."""
    if n == 1:
        return np.array([hi], np.int64)
    return np.rint(np.exp(np.linspace(math.log(lo), math.log(hi), n))).astype(np.int64)


def _up(a, b):
    return -(-a // b)


def _i32(a):
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.int32)).cuda()


def _cache(c, g, pages, lens, refs, layers):
    shape = (layers, len(refs), c["kv_heads"], c["page"], c["head_dim"])
    return {"pool_k": _normal(g, shape, 1.0, _dtype(c)),
            "pool_v": _normal(g, shape[:3] + (c["head_dim"], c["page"]), 1.0, _dtype(c)), "pages": _i32(pages),
            "lens": _i32(lens), "refs": _i32(refs), "status": torch.zeros(1, dtype=torch.int32, device="cuda")}


def _branches(c):
    """(prompt, length, new tokens) of every slot: each prompt in a slot of its own, without new tokens, then its
    branches, which end at different lengths."""
    P, N, n = c["prompts"], c["branches"], c["n"]
    root = _spread(P, max(1, c["prompt_len"] // 2), c["prompt_len"])
    tail = np.maximum(_spread(N, 1, c["tail"]), n)
    prompt, lens, new = [], [], []
    for p in range(P):
        prompt += [p] * (1 + N)
        lens += [int(root[p])] + [int(root[p] + tail[(j * 5 + p) % N]) for j in range(N)]
        new += [0] + [max(1, n - j % 3) for j in range(N)]
    return root, np.array(prompt), np.array(lens), np.array(new)


def _shared_state(c, g, rng):
    ps = c["page"]
    root, prompt, lens, new = _branches(c)
    S, width = len(lens), _up(int(lens.max()), ps) + 1
    n_pages = int(_up(root, ps).sum() + sum(_up(int(L), ps) - int(root[p]) // ps for L, p in zip(lens, prompt))) + 3
    free = list(rng.permutation(n_pages))
    # the pages that a prompt fills are shared; a page that it fills in part was copied for each branch
    whole = [[free.pop() for _ in range(int(L) // ps)] for L in root]
    pages, refs = np.full((S, width), -1, np.int64), np.zeros(n_pages, np.int64)
    for s, (p, L) in enumerate(zip(prompt, lens)):
        table = whole[p] + [free.pop() for _ in range(_up(int(L), ps) - len(whole[p]))]
        pages[s, :len(table)] = table
        np.add.at(refs, table, 1)
    order = rng.permutation(S)
    s = _cache(c, g, pages[order], lens[order], refs, c["layers"])
    hq, hk, d, rows = c["heads"], c["kv_heads"], c["head_dim"], S * c["n"]
    qkv = _normal(g, (c["layers"], rows, hq + 2 * hk, d), 1.0, _dtype(c))  # the fused projections' rows
    qkv[:, :, :hq] *= 2.0
    s |= {"group": _i32(prompt[order]), "new": _i32(new[order]), "q": [qkv[layer, :, :hq] for layer in range(c["layers"])],
          "out": torch.zeros(c["layers"], rows, hq * d, dtype=_dtype(c), device="cuda"),
          "lse": torch.zeros(c["layers"], rows, hq, device="cuda")}
    # free pages hold what an earlier sequence left there
    gone = (s["refs"] == 0).nonzero().view(-1)
    s["pool_k"][:, gone] = float("nan")
    s["pool_v"][:, gone] = float("nan")
    return s


def _rows(c):
    """(lengths, new tokens) of a rotate case's sequences, unordered."""
    S, n = c["seqs"], c["n"]
    new = _spread(S, max(1, n // 4), n)
    return np.maximum(_spread(S, max(1, c["max_len"] // 64), c["max_len"]), new), new


# kind, factor, trained context, turns below and above which a frequency is scaled in full or not at all
SCALING = {"none": None, "linear": ("linear", 4.0, 8192, 1.0, 4.0), "base": ("base", 4.0, 8192, 1.0, 4.0),
           "by_rotations": ("by_rotations", 8.0, 8192, 1.0, 4.0), "by_index": ("by_index", 16.0, 8192, 1.0, 32.0)}
THETA, EPS = 500000.0, 1e-5


def _rotate_state(c, g, rng):
    S, n, hq, hk, d, ps = c["seqs"], c["n"], c["heads"], c["kv_heads"], c["head_dim"], c["page"]
    lens, new = _rows(c)
    order = rng.permutation(S)
    lens, new = lens[order], new[order]
    used = _up(lens, ps)
    n_pages = int(used.sum()) + 3
    ids = rng.permutation(n_pages)
    pages, refs = np.full((S, int(used.max())), -1, np.int64), np.zeros(n_pages, np.int64)
    at = np.concatenate([[0], np.cumsum(used)])
    for s in range(S):
        pages[s, :used[s]] = ids[at[s]:at[s + 1]]
    refs[ids[:at[-1]]] = 1
    s = _cache(c, g, pages, lens, refs, 2)
    qkv = _normal(g, (S * n, hq + 2 * hk, d), 1.0, _dtype(c))
    s |= {"new": _i32(new), "q": qkv[:, :hq], "k": qkv[:, hq:hq + hk], "v": qkv[:, hq + hk:], "positions": None,
          "q_norm": None, "k_norm": None, "out": torch.zeros(S * n, hq, d, dtype=_dtype(c), device="cuda")}
    if c["norms"]:
        s["q_norm"], s["k_norm"] = (1.0 + 0.2 * torch.randn(d, generator=g, device="cuda") for _ in range(2))
    if c["ahead"]:  # positions that go on from a context which this cache no longer holds
        first = torch.from_numpy(rng.integers(c["ahead"] // 2, c["ahead"], S)).cuda()
        s["positions"] = (first[:, None] + torch.arange(n, device="cuda")).view(-1).to(torch.int32)
    return s


def _sample_state(c, g, rng):
    R, V = c["rows"], c["vocab"]
    # a few likely tokens over noise
    z = torch.randn(R, V, generator=g, device="cuda").mul_(2.0)
    likely = torch.randint(0, V, (R, 40), generator=g, device="cuda")
    z.scatter_add_(1, likely, torch.rand(R, 40, generator=g, device="cuda") * 10.0)
    if c["banned"]:  # ids that a grammar forbids
        z[torch.rand(R, V, generator=g, device="cuda") < 0.3] = -math.inf
    T, k = np.full(R, c["T"], np.float32), np.full(R, c["top_k"])
    p, m = np.full(R, c["top_p"], np.float32), np.full(R, c["min_p"], np.float32)
    if c["mix"]:  # every fourth row as the case says; the others without one of the limits, or greedy
        turn = rng.permutation(R) % 4
        k[turn == 1], p[turn == 1], m[turn == 2], T[turn == 3] = 0, 1.0, 0.0, 0.0
    f32 = lambda a: torch.from_numpy(a).cuda()  # noqa: E731
    return {"z": z, "u": torch.rand(R, generator=g, device="cuda"), "T": f32(T),
            "top_k": _i32(k) if c["top_k"] else None, "top_p": f32(p) if c["top_p"] < 1 else None,
            "min_p": f32(m) if c["min_p"] else None}


def prepare(case, seed):
    make = {"shared": _shared_state, "rotate": _rotate_state, "sample": _sample_state}[case["kind"]]
    s = make(case, _gen(seed), np.random.default_rng(int(seed) * 51769 + 11))
    s["case"] = case
    return s


# --------------------------------------------------------------------- runs --
LAYER = 1  # of the two layers that a rotate case holds


def _handle(s):
    """The framework's view of the cache and the workspaces, made once as a program keeps them."""
    import paper_2607_20791_amd as rgd
    c = s["case"]
    if "handle" not in s:
        empty = lambda n: torch.empty(max(n, 1), dtype=torch.uint8, device="cuda")  # noqa: E731
        if c["kind"] == "sample":
            s["handle"], R = None, c["rows"]
            s["ws"] = empty(rgd.sample_truncated_workspace_bytes(R, c["vocab"]))
            s["token"] = torch.empty(R, dtype=torch.int32, device="cuda")
            s["logp"] = torch.empty(R, dtype=torch.float32, device="cuda")
            return rgd, None
        s["handle"] = rgd.PagedCache(s["pool_k"], s["pool_v"], s["pages"], s["lens"], s["refs"], s["status"])
        if c["kind"] == "shared":
            s["plan"] = empty(rgd.paged_share_bytes(s["handle"], c["n"], c["heads"]))
            s["ws"] = empty(rgd.paged_attention_shared_workspace_bytes(s["handle"], c["n"], c["heads"]))
            s["shared"] = torch.empty(len(s["lens"]), dtype=torch.int32, device="cuda")
        else:
            how = SCALING[c["scaling"]]
            s["rotary"] = rgd.Rotary(c["dims"], THETA, interleaved=c["layout"] == "interleaved",
                                     scaling=how and rgd.RotaryScaling(*how))
    return rgd, s["handle"]


def run(state):
    return {"shared": _shared, "rotate": _rotate, "sample": _sample}[state["case"]["kind"]](state, state["case"])


def _common(s, c):
    """Positions that every sequence's group reads once: the whole pages in front of its members' new tokens that all
    members with new tokens have in the same places."""
    pages, new, ps = s["pages"].long(), s["new"].long(), c["page"]
    S, width = pages.shape
    active = new > 0
    label = s["group"].long()
    first = torch.full((S,), S, device="cuda").scatter_reduce(0, label, torch.where(active, torch.arange(S, device="cuda"), S), "amin")
    like = pages[first[label].clamp(max=S - 1)]
    run_of = ((pages == like).long().cumprod(1)).sum(1)
    most = torch.minimum(run_of, (s["lens"].long() - new).clamp(min=0) // ps)
    least = torch.full((S,), width, device="cuda").scatter_reduce(0, label, torch.where(active, most, width), "amin")
    members = torch.zeros(S, dtype=torch.long, device="cuda").scatter_add(0, label, active.long())
    return torch.where(active & (members[label] > 1), least[label] * ps, 0).to(torch.int32)


def _shared(s, c):
    n, hq, hk, d, S = c["n"], c["heads"], c["kv_heads"], c["head_dim"], len(s["lens"])
    if own:
        rgd, cache = _handle(s)
        rgd.paged_share(cache, n, s["new"], hq, s["group"], s["plan"], s["shared"])
        for layer in range(c["layers"]):
            rgd.paged_attention_shared(cache, layer, s["q"][layer], n, s["plan"], s["ws"], s["out"][layer], s["lse"][layer])
        return s["shared"], s["out"], s["lse"]
    lens, new = s["lens"].long(), s["new"].long()
    L = s["pages"].shape[1] * c["page"]
    ids = s["pages"].long().clamp(min=0)
    there = (torch.arange(L, device="cuda") < lens[:, None])[:, None, :, None]
    end = lens[:, None] - new[:, None] + torch.arange(n, device="cuda") + 1  # positions that token i sees
    seen = (torch.arange(L, device="cuda") < end[:, :, None])[:, None, None].expand(S, hk, hq // hk, n, L).reshape(S, hk, -1, L)
    row = (torch.arange(n, device="cuda") < new[:, None]).view(-1, 1)
    for layer in range(c["layers"]):
        k = s["pool_k"][layer][ids].permute(0, 2, 1, 3, 4).reshape(S, hk, L, d).float()
        v = s["pool_v"][layer][ids].permute(0, 2, 1, 4, 3).reshape(S, hk, L, d).float()
        k, v = torch.where(there, k, 0.0), torch.where(there, v, 0.0)
        q = s["q"][layer].float().reshape(S, n, hk, hq // hk, d).permute(0, 2, 3, 1, 4).reshape(S, hk, hq // hk * n, d)
        a = torch.matmul(q, k.transpose(2, 3).contiguous()) / math.sqrt(d)
        a = torch.where(seen, a, -math.inf)
        top = a.amax(-1, keepdim=True).clamp(min=-3e38)
        e = torch.exp(a - top)
        z = e.sum(-1, keepdim=True)
        o = torch.matmul(e, v) / torch.where(z > 0, z, 1.0)
        lse = (top + torch.log(z)).view(S, hk, hq // hk, n).permute(0, 3, 1, 2).reshape(S * n, hq)
        o = o.view(S, hk, hq // hk, n, d).permute(0, 3, 1, 2, 4).reshape(S * n, hq * d)
        s["out"][layer].copy_(torch.where(row, o.to(s["out"].dtype), s["out"][layer]))
        s["lse"][layer].copy_(torch.where(row, lse, s["lse"][layer]))
    return _common(s, c), s["out"], s["lse"]


def _frequencies(c):
    """Radians per position of each pair, and the factor of cosine and sine, in 64 bits."""
    dims, theta = c["dims"], THETA
    j = torch.arange(dims // 2, dtype=torch.float64, device="cuda")
    if SCALING[c["scaling"]] is None:
        return theta ** (-2.0 * j / dims), 1.0
    kind, factor, context, low, high = SCALING[c["scaling"]]
    if kind == "base":
        return (theta * factor ** (dims / (dims - 2.0))) ** (-2.0 * j / dims), 1.0
    f = theta ** (-2.0 * j / dims)
    if kind == "linear":
        return f / factor, 1.0
    if kind == "by_rotations":
        kept = ((context * f / (2 * math.pi) - low) / (high - low)).clamp(0, 1)
        return f * ((1 - kept) / factor + kept), 1.0
    index = lambda turns: dims * math.log(context / (2 * math.pi * turns)) / (2 * math.log(theta))  # noqa: E731
    a, b = max(math.floor(index(high)), 0), min(math.ceil(index(low)), dims - 1)
    scaled = ((j - a) / max(b - a, 1e-3)).clamp(0, 1)
    return f * (scaled / factor + 1 - scaled), 0.1 * math.log(factor) + 1


def _turn(x, gain, cos, sin, c):
    """Head norm and rotation of rows [n][heads][d] in 32 bits."""
    x = x.float()
    if gain is not None:
        x = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS) * gain
    dims = c["dims"]
    if c["layout"] == "half":
        a, b = x[..., :dims // 2], x[..., dims // 2:dims]
        turned = torch.cat([a * cos - b * sin, b * cos + a * sin], -1)
    else:
        a, b = x[..., 0:dims:2], x[..., 1:dims:2]
        turned = torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2)
    return torch.cat([turned, x[..., dims:]], -1)


def _places(s, c):
    """(rows with a token, their positions in the cache, pages, slots)."""
    i = torch.arange(c["n"], device="cuda")
    lens, new = s["lens"].long(), s["new"].long()
    at = lens[:, None] - new[:, None] + i
    row = (i < new[:, None]).view(-1)
    page = s["pages"].long().gather(1, (at // c["page"]).clamp(0, s["pages"].shape[1] - 1)).view(-1)[row]
    return row, at.view(-1), page, (at % c["page"]).view(-1)[row]


def _rotate(s, c):
    if own:
        rgd, cache = _handle(s)
        rgd.paged_append_rotated(cache, LAYER, s["q"], s["k"], s["v"], c["n"], s["rotary"], s["out"], n_new=s["new"],
                                 positions=s["positions"], q_norm=s["q_norm"], k_norm=s["k_norm"], eps=EPS)
        return s["out"], s["pool_k"], s["pool_v"]
    row, at, page, slot = _places(s, c)
    freq, scale = _frequencies(c)
    pos = at if s["positions"] is None else s["positions"].long()
    angle = pos.double()[:, None] * freq
    cos, sin = (torch.cos(angle) * scale).float()[:, None], (torch.sin(angle) * scale).float()[:, None]
    q, k = _turn(s["q"], s["q_norm"], cos, sin, c), _turn(s["k"], s["k_norm"], cos, sin, c)
    s["out"].copy_(torch.where(row[:, None, None], q.to(s["out"].dtype), s["out"]))
    s["pool_k"][LAYER][page, :, slot] = k[row].to(s["out"].dtype)
    s["pool_v"][LAYER][page, :, :, slot] = s["v"][row]
    return s["out"], s["pool_k"], s["pool_v"]


def _sample(s, c):
    if own:
        rgd, _ = _handle(s)
        rgd.sample_truncated(s["z"], s["u"], s["ws"], s["token"], T=s["T"], top_k=s["top_k"], top_p=s["top_p"],
                             min_p=s["min_p"], logp=s["logp"])
        return s["token"], s["logp"]
    R, V = s["z"].shape
    z, order = torch.sort(s["z"].double(), dim=1, descending=True, stable=True)
    z = z - z[:, :1]
    rank = torch.arange(V, device="cuda")
    T = s["T"].double()[:, None]
    # at temperature 0 the first maximum has everything
    w = torch.where(T > 0, torch.exp(z / torch.where(T > 0, T, 1.0)), (rank == 0).double())
    kept = w > 0
    if s["top_k"] is not None:
        k = s["top_k"].long()[:, None]
        kept &= (k <= 0) | (rank < k)
    if s["top_p"] is not None:
        p = s["top_p"].double()[:, None]
        part = torch.where(kept, w, 0.0)
        upto = part.cumsum(1)
        kept &= (upto - part < p * upto[:, -1:]) | (p >= 1) | (rank == 0)
    if s["min_p"] is not None:
        m = s["min_p"].double()[:, None]
        kept &= (z >= T * torch.log(m)) | (m <= 0)
    w = torch.zeros_like(w).scatter(1, order, torch.where(kept, w, 0.0))
    upto = w.cumsum(1)
    token = (upto <= s["u"].double()[:, None] * upto[:, -1:]).sum(1, keepdim=True).clamp(max=V - 1)
    logp = torch.log(w.gather(1, token) / upto[:, -1:])
    return token[:, 0].to(torch.int32), logp[:, 0].float()


# --------------------------------------------------------------------- work --
def work(case):
    c, kind = case, case["kind"]
    if kind == "sample":
        return {"bytes": 4 * c["rows"] * c["vocab"] + 28 * c["rows"], "flops": 4 * c["rows"] * c["vocab"]}
    hq, hk, d, size = c["heads"], c["kv_heads"], c["head_dim"], _size(c)
    if kind == "rotate":
        _, new = _rows(c)
        return {"bytes": 2 * int(new.sum()) * (hq + 2 * hk) * d * size, "flops": 8 * int(new.sum()) * (hq + hk) * d}
    root, prompt, lens, new = _branches(c)
    once = 0  # positions that have to be read
    for p in range(c["prompts"]):
        mine = (prompt == p) & (new > 0)
        # pages that every branch holds, in front of the new tokens of each
        shared = min(int(root[p]), int((lens - new)[mine].min())) // c["page"] * c["page"] if mine.sum() > 1 else 0
        once += shared + int((lens[mine] - shared).sum())
    rows = int(new.sum())
    seen = int((new * lens - new * (new - 1) // 2).sum())
    return {"bytes": c["layers"] * (once * hk * d * 2 * size + rows * hq * (2 * d * size + 4)) + 4 * len(lens) * (int(lens.max()) // c["page"] + 5),
            "flops": 4 * c["layers"] * hq * d * seen}


# -------------------------------------------------------------------- exact --
def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "shared":
        return _exact_shared(s, case)
    if case["kind"] == "rotate":
        return _exact_rotate(s, case)
    return _exact_sample(s, case)


def _exact_shared(s, c):
    n, hq, hk, d, ps = c["n"], c["heads"], c["kv_heads"], c["head_dim"], c["page"]
    G = hq // hk
    out, lse = s["out"].double(), s["lse"].double()
    lens, new = s["lens"].tolist(), s["new"].tolist()
    for layer in range(c["layers"]):
        q = s["q"][layer].double().view(-1, n, hk, G, d)
        for b, (L, m) in enumerate(zip(lens, new)):
            if m == 0:
                continue
            ids = s["pages"][b, :_up(L, ps)].long()
            keys = s["pool_k"][layer, ids].transpose(0, 1).reshape(hk, -1, d)[:, :L].double()
            vals = s["pool_v"][layer, ids].transpose(2, 3).transpose(0, 1).reshape(hk, -1, d)[:, :L].double()
            for i in range(m):
                t = L - m + i + 1
                a = torch.bmm(q[b, i], keys[:, :t].transpose(1, 2).contiguous()) * d ** -0.5
                l = torch.logsumexp(a, 2)
                o = torch.bmm(torch.exp(a - l[..., None]), vals[:, :t].contiguous())
                lse[layer, b * n + i] = l.view(-1)
                out[layer, b * n + i] = o.view(-1)
    return None, out, lse


def _exact_rotate(s, c):
    """A pair as a complex number, times e^(i angle)."""
    row, at, page, slot = _places(s, c)
    dims, theta = c["dims"], THETA
    how = SCALING[c["scaling"]]
    freq, scale = [], 1.0
    for j in range(dims // 2):
        f = theta ** (-2.0 * j / dims)
        if how is not None:
            kind, factor, context, low, high = how
            if kind == "linear":
                f /= factor
            elif kind == "base":
                f = (theta * factor ** (dims / (dims - 2.0))) ** (-2.0 * j / dims)
            elif kind == "by_rotations":
                turns = context * f / (2 * math.pi)
                f = f / factor if turns <= low else f if turns >= high else \
                    f / factor + (f - f / factor) * (turns - low) / (high - low)
            else:
                where = [dims * math.log(context / (2 * math.pi * r)) / (2 * math.log(theta)) for r in (high, low)]
                a, b = max(math.floor(where[0]), 0), min(math.ceil(where[1]), dims - 1)
                mixed = min(max((j - a) / max(b - a, 1e-3), 0.0), 1.0)
                f = f + mixed * (f / factor - f)
                scale = 1 + math.log(factor) / 10
        freq.append(f)
    pos = at if s["positions"] is None else s["positions"].long()
    turn = torch.polar(torch.full((1,), scale, dtype=torch.float64, device="cuda"),
                       torch.outer(pos.double(), torch.tensor(freq, dtype=torch.float64, device="cuda")))[:, None]
    res = []
    for x, gain in ((s["q"], s["q_norm"]), (s["k"], s["k_norm"])):
        x = x.double().clone()
        if gain is not None:
            x = x / torch.sqrt(torch.mean(x ** 2, -1, keepdim=True) + EPS) * gain.double()
        first, second = (slice(0, dims // 2), slice(dims // 2, dims)) if c["layout"] == "half" else \
            (slice(0, dims, 2), slice(1, dims, 2))
        pair = torch.complex(x[..., first].contiguous(), x[..., second].contiguous()) * turn
        x[..., first], x[..., second] = pair.real, pair.imag
        res.append(x)
    out, pool = s["out"].double(), s["pool_k"].double()
    out[row] = res[0][row]
    pool[LAYER][page, :, slot] = res[1][row]
    return out, pool, None


def _exact_sample(s, c):
    zs, us = s["z"].cpu().numpy().astype(np.float64), s["u"].cpu().numpy().astype(np.float64)
    at = lambda name, r, off: off if s[name] is None else float(s[name][r])  # noqa: E731
    tokens, logp = np.zeros(len(zs), np.int32), np.zeros(len(zs))
    for r, z in enumerate(zs):
        T = at("T", r, 1.0)
        if T <= 0:
            tokens[r] = int(np.argmax(z))
            continue
        order = np.argsort(-z, kind="stable")
        w = np.exp((z - z.max()) / T)
        k = int(at("top_k", r, 0))
        ids = order[:k] if k > 0 else order
        ids = ids[w[ids] > 0]
        p, m = at("top_p", r, 1.0), at("min_p", r, 0.0)
        if p < 1:
            run_sum = np.cumsum(w[ids])
            ids = ids[:1 + int(np.searchsorted(run_sum, p * run_sum[-1]))]
        if m > 0:
            ids = ids[z[ids] - z.max() >= T * math.log(m)]
        ids = np.sort(ids)
        run_sum = np.cumsum(w[ids])
        tokens[r] = t = ids[min(int(np.searchsorted(run_sum, us[r] * run_sum[-1], side="right")), len(ids) - 1)]
        logp[r] = (z[t] - z.max()) / T - math.log(math.fsum(w[ids]))
    return tokens, logp
