"""Measured cases of the paged cache's operators and of the verification of drafted tokens.

Each case is a plain dict; `prepare` builds what a serving program holds before the call (pools, page tables,
lengths, logits), `run` makes one pass, either in plain torch operations or (with `own`) through the entry points of
`paper_2607_20791_amd`, and `exact` computes the same outputs in 64 bits.

Kinds:
  attention  new tokens of sequences of uneven lengths over their pages, one layer
  append     the new tokens' K and V rows put into the pages, one layer
  branch     one turn of sampled branches: trimmed or forked from their prompt again, pages for the next tokens
             reserved, shared partial pages copied, all layers
  compact    live pages moved to the lowest ids, all layers
  verify     drafted tokens checked against the target's truncated distribution, the next token drawn

Lengths are spread over their range by the case alone (the seed orders them), so that a case's work is known.
"""
import math

import numpy as np
import torch

own = False


def listed():
    return [
        # one request's next token over a short cache: launches and latency
        {"name": "attention-1x1-p512", "kind": "attention", "seqs": 1, "n": 1, "heads": 32, "kv_heads": 8,
         "head_dim": 128, "dtype": "bf16", "page": 16, "max_len": 512, "spread": "full"},
        # a batch of requests of every length
        {"name": "attention-64x1-p8192", "kind": "attention", "seqs": 64, "n": 1, "heads": 32, "kv_heads": 8,
         "head_dim": 128, "dtype": "bf16", "page": 16, "max_len": 8192, "spread": "ragged"},
        # one very long request
        {"name": "attention-1x1-p131072", "kind": "attention", "seqs": 1, "n": 1, "heads": 32, "kv_heads": 8,
         "head_dim": 128, "dtype": "bf16", "page": 64, "max_len": 131072, "spread": "full"},
        # four drafted tokens and the one before them, ragged counts
        {"name": "attention-32x5-p4096", "kind": "attention", "seqs": 32, "n": 5, "heads": 32, "kv_heads": 8,
         "head_dim": 128, "dtype": "bf16", "page": 16, "max_len": 4096, "spread": "ragged"},
        # the small fp32 decoder's heads at odd lengths
        {"name": "attention-f32-16x1-p999", "kind": "attention", "seqs": 16, "n": 1, "heads": 4, "kv_heads": 2,
         "head_dim": 64, "dtype": "f32", "page": 16, "max_len": 999, "spread": "ragged"},
        # one step's tokens of 64 branches
        {"name": "append-64x1", "kind": "append", "seqs": 64, "n": 1, "heads": 32, "kv_heads": 8, "head_dim": 128,
         "dtype": "bf16", "page": 16, "max_len": 2048},
        # eight prompts in pieces of up to 1000 tokens
        {"name": "append-8x1000", "kind": "append", "seqs": 8, "n": 1000, "heads": 32, "kv_heads": 8,
         "head_dim": 128, "dtype": "bf16", "page": 16, "max_len": 4096},
        # 32 prompts with 8 branches each, half of them forked again
        {"name": "branch-32x8", "kind": "branch", "prompts": 32, "branches": 8, "layers": 8, "kv_heads": 8,
         "head_dim": 128, "dtype": "bf16", "page": 16, "max_len": 1024, "grow": 5},
        # a third of a large pool lives, in scattered pages
        {"name": "compact-16384", "kind": "compact", "seqs": 64, "layers": 4, "pages": 16384, "kv_heads": 8,
         "head_dim": 128, "dtype": "bf16", "page": 16, "max_len": 3000},
        # one request, four drafts of a small model
        {"name": "verify-1x4", "kind": "verify", "seqs": 1, "k": 4, "vocab": 128256, "T": 1.0, "min_p": 0.1,
         "draft": "logits"},
        # a batch of them at the largest vocabulary and a high temperature
        {"name": "verify-64x4", "kind": "verify", "seqs": 64, "k": 4, "vocab": 152064, "T": 2.0, "min_p": 0.05,
         "draft": "logits"},
        # greedy probes as drafts: tokens without probabilities of their own
        {"name": "verify-32x15-probe", "kind": "verify", "seqs": 32, "k": 15, "vocab": 128256, "T": 1.5,
         "min_p": 0.1, "draft": "tokens"},
    ]


def _log(rng, lo, hi):
    """An integer spread over the logarithm of [lo, hi]."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["attention", "attention", "append", "branch", "compact", "verify", "verify"])
    dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
    page = rng.choice([16, 16, 32, 64])
    dim = rng.choice([64, 128] if dtype == "bf16" else [32, 64, 128])
    hk = rng.choice([1, 2, 4, 8])
    if kind == "attention":
        seqs = _log(rng, 1, 64)
        most = min(131072, 131072 * 8 * 128 // (seqs * hk * dim) // (1 if dtype == "bf16" else 2))
        return {"kind": kind, "seqs": seqs, "n": rng.choice([1, 1, 1, rng.randint(2, 8)]),
                "heads": hk * rng.choice([1, 2, 4, 8]), "kv_heads": hk, "head_dim": dim, "dtype": dtype,
                "page": page, "max_len": _log(rng, 1, most), "spread": rng.choice(["full", "ragged", "ragged"])}
    if kind == "append":
        seqs = _log(rng, 1, 64)
        n = rng.choice([1, rng.randint(2, 8), _log(rng, 9, 1000)])
        return {"kind": kind, "seqs": seqs, "n": n, "heads": hk * rng.choice([1, 2, 4, 8]), "kv_heads": hk,
                "head_dim": dim, "dtype": dtype, "page": page, "max_len": _log(rng, max(n, 16), 4096)}
    if kind == "branch":
        prompts = _log(rng, 1, 32)
        return {"kind": kind, "prompts": prompts, "branches": _log(rng, 1, 256 // prompts),
                "layers": rng.choice([1, 2, 4, 8]), "kv_heads": hk, "head_dim": dim, "dtype": dtype, "page": page,
                "max_len": _log(rng, 40, 1024), "grow": rng.randint(1, 32)}
    if kind == "compact":
        return {"kind": kind, "seqs": _log(rng, 1, 64), "layers": rng.choice([1, 2, 4]),
                "pages": _log(rng, 200, 8192 * 16 // page // (1 if dtype == "bf16" else 2)), "kv_heads": hk,
                "head_dim": dim, "dtype": dtype, "page": page, "max_len": _log(rng, 100, 3000)}
    draft = rng.choice(["logits", "logits", "tokens"])
    k = rng.randint(1, 8) if draft == "logits" else rng.randint(1, 15)
    return {"kind": kind, "seqs": _log(rng, 1, min(64, 64 * 9 // (2 * k + 1 if draft == "logits" else k + 1))),
            "k": k, "vocab": _log(rng, 8000, 152064), "T": rng.choice([0.0, 0.7, 1.0, 1.5, 2.0]),
            "min_p": rng.choice([0.0, 0.05, 0.1, 0.2]), "draft": draft}


# ------------------------------------------------------------------- inputs --
def _dtype(c):
    return torch.bfloat16 if c["dtype"] == "bf16" else torch.float32


def _size(c):
    return 2 if c["dtype"] == "bf16" else 4


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(int(seed) * 7919 + 17)


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


def _lengths(c):
    """(lengths, new tokens) of a case's sequences, unordered."""
    S, n, hi = c["seqs"], c["n"], c["max_len"]
    lens = np.full(S, hi, np.int64) if c.get("spread") == "full" else _spread(S, 1, hi)
    new = np.full(S, n, np.int64) if c["kind"] == "attention" else _spread(S, max(1, n // 4), n)
    if c["kind"] == "append":
        lens = np.maximum(lens, new)
    elif S >= 8:
        lens[0] = new[0] = 0  # an empty slot
        new[1::3] = np.maximum(1, n - 1)
    return lens, np.minimum(new, lens)


def _up(a, b):
    return -(-a // b)


def _i32(a):
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.int32)).cuda()


def _pools(c, g, layers, n_pages):
    shape = (layers, n_pages, c["kv_heads"], c["page"], c["head_dim"])
    return _normal(g, shape, 1.0, _dtype(c)), _normal(g, shape[:3] + (c["head_dim"], c["page"]), 1.0, _dtype(c))


def _cache(c, g, rng, lens, layers, extra):
    """A cache whose sequences hold pages of their own, in a random order, and `extra` free ones."""
    ps, S = c["page"], len(lens)
    used = _up(lens, ps)
    width = max(1, int(used.max()))
    n_pages = int(used.sum()) + extra
    order = rng.permutation(n_pages)
    pages = np.full((S, width), -1, np.int64)
    refs = np.zeros(n_pages, np.int64)
    at = 0
    for s in range(S):
        pages[s, :used[s]] = order[at:at + used[s]]
        at += int(used[s])
    refs[order[:at]] = 1
    pk, pv = _pools(c, g, layers, n_pages)
    return {"pool_k": pk, "pool_v": pv, "pages": _i32(pages), "lens": _i32(lens), "refs": _i32(refs),
            "status": torch.zeros(1, dtype=torch.int32, device="cuda")}


def _stale(s, c):
    """What a cache that has been in use holds where no token is visible: free pages and the rest of last pages are NaN."""
    ps, lens = c["page"], s["lens"].long()
    free = (s["refs"] == 0).nonzero().view(-1)
    s["pool_k"][:, free] = float("nan")
    s["pool_v"][:, free] = float("nan")
    part = ((lens > 0) & (lens % ps != 0)).nonzero().view(-1)
    last = s["pages"][part, lens[part] // ps].long()
    gone = torch.arange(ps, device="cuda") >= (lens[part] % ps)[:, None]
    nan = torch.tensor(float("nan"), dtype=s["pool_k"].dtype, device="cuda")
    s["pool_k"][:, last] = torch.where(gone[None, :, None, :, None], nan, s["pool_k"][:, last])
    s["pool_v"][:, last] = torch.where(gone[None, :, None, None, :], nan, s["pool_v"][:, last])


def _branch_state(c, g, rng):
    """Prompts in slots 0, 1 + N, ...; behind each its N branches.  Even branches go on from tails of their own; odd
    ones are forked from the prompt again in the turn that is measured."""
    P, N, ps, grow = c["prompts"], c["branches"], c["page"], c["grow"]
    S = P * (1 + N)
    lens, keep, add = np.zeros(S, np.int64), np.full(S, -1, np.int64), np.zeros(S, np.int64)
    parent = np.arange(S)
    width = _up(c["max_len"] + 3 * grow, ps) + 1
    tables = [[] for _ in range(S)]
    root_len = _spread(P, max(1, c["max_len"] // 4), c["max_len"])
    n_pages = int(sum(_up(root_len, ps))) + S * (_up(3 * grow + ps, ps) + 1)
    order = list(rng.permutation(n_pages))
    for p in range(P):
        r = p * (1 + N)
        L = int(root_len[p])
        lens[r], tables[r] = L, [order.pop() for _ in range(_up(L, ps))]
        for j in range(N):
            s = r + 1 + j
            lens[s] = L + 1 + (j * 7) % (2 * grow)
            full = L // ps
            tables[s] = tables[r][:full] + [order.pop() for _ in range(_up(int(lens[s]), ps) - full)]
            add[s] = 1 + (j * 3) % grow
            if j % 2:
                parent[s] = r
            else:
                keep[s] = L + (j * 5) % grow if lens[s] >= L + (j * 5) % grow else lens[s]
    pages, refs = np.full((S, width), -1, np.int64), np.zeros(n_pages, np.int64)
    for s in range(S):
        pages[s, :len(tables[s])] = tables[s]
        np.add.at(refs, tables[s], 1)
    pk, pv = _pools(c, g, c["layers"], n_pages)
    return {"pool_k": pk, "pool_v": pv, "pages": _i32(pages), "lens": _i32(lens), "refs": _i32(refs),
            "status": torch.zeros(1, dtype=torch.int32, device="cuda"), "parent": _i32(parent), "keep": _i32(keep),
            "grow": _i32(add)}


def _drafts(c):
    k = np.full(c["seqs"], c["k"], np.int64)
    k[3::4] = c["k"] // 2
    return k


def _verify_state(c, g, rng):
    S, K, V = c["seqs"], c["k"], c["vocab"]
    # a few likely tokens over noise; the small model's logits are near the target's
    target = torch.randn(S, K + 1, V, generator=g, device="cuda").mul_(2.0)
    likely = torch.randint(0, V, (S, K + 1, 40), generator=g, device="cuda")
    target.scatter_add_(2, likely, torch.rand(S, K + 1, 40, generator=g, device="cuda") * 10.0)
    s = {"target": target, "n_draft": _i32(rng.permutation(_drafts(c))),
         "u": torch.rand(S, K + 1, generator=g, device="cuda"), "draft": None}
    if c["draft"] == "logits":
        near = target[:, :K].contiguous()
        near += torch.randn(S, K, V, generator=g, device="cuda").mul_(0.5)
        s["draft"] = near
        # the drafts are draws from the small model's truncated distribution
        noise = torch.rand(S, K, V, generator=g, device="cuda").clamp_(1e-30).log_().neg_().log_()
        noise = near / max(c["T"], 1e-3) - noise
        if c["min_p"] > 0:
            low = near.amax(-1, keepdim=True) + c["T"] * math.log(c["min_p"])
            noise = torch.where(near >= low, noise, -math.inf)
        s["tokens"] = noise.argmax(-1).to(torch.int32)
    else:
        s["tokens"] = target[:, :K].argmax(-1).to(torch.int32)
    return s


def prepare(case, seed):
    c, g = case, _gen(seed)
    rng = np.random.default_rng(int(seed) * 104729 + 3)
    kind = c["kind"]
    if kind == "verify":
        s = _verify_state(c, g, rng)
    elif kind == "branch":
        s = _branch_state(c, g, rng)
    elif kind == "compact":
        S, ps = c["seqs"], c["page"]
        lens = rng.permutation(np.minimum(_spread(S, 20, c["max_len"]), max(1, c["pages"] // 2 // S * ps)))
        s = _cache(c, g, rng, lens, c["layers"], c["pages"] - int(_up(lens, ps).sum()))
        s["before"] = (s["pages"].clone(), s["refs"].clone())
    else:
        lens, new = _lengths(c)
        order = rng.permutation(len(lens))
        s = _cache(c, g, rng, lens[order], 2, 3)
        S, n, hq, hk, d = c["seqs"], c["n"], c["heads"], c["kv_heads"], c["head_dim"]
        s["new"] = _i32(new[order])
        qkv = _normal(g, (S * n, hq + 2 * hk, d), 1.0, _dtype(c))  # the fused projection's rows
        s["q"], s["k"], s["v"] = qkv[:, :hq], qkv[:, hq:hq + hk], qkv[:, hq + hk:]
        if kind == "attention":
            s["q"] *= 2.0
            s["out"] = torch.zeros(S * n, hq * d, dtype=_dtype(c), device="cuda")
            s["lse"] = torch.zeros(S * n, hq, device="cuda")
            _stale(s, c)
    s["case"] = c
    return s


# --------------------------------------------------------------------- runs --
LAYER = 1  # of the two layers that attention and append hold


def _outputs(s):
    return {k: s[k] for k in ("pages", "lens", "refs", "status", "pool_k", "pool_v")}


def _handle(s):
    """The framework's view of the cache and its workspace, made once as a program keeps them."""
    import paper_2607_20791_amd as rgd
    if "handle" not in s:
        s["handle"] = rgd.PagedCache(s["pool_k"], s["pool_v"], s["pages"], s["lens"], s["refs"], s["status"])
        c = s["case"]
        n = (rgd.paged_attention_workspace_bytes(s["handle"], c["n"], c["heads"]) if c["kind"] == "attention"
             else rgd.paged_workspace_bytes(s["handle"]))
        s["ws"] = torch.empty(max(n, 1), dtype=torch.uint8, device="cuda")
    return rgd, s["handle"], s["ws"]


def run(state):
    s, c = state, state["case"]
    return {"attention": _attention, "append": _append, "branch": _branch, "compact": _compact,
            "verify": _verify}[c["kind"]](s, c)


def _attention(s, c):
    n, hq, hk, d = c["n"], c["heads"], c["kv_heads"], c["head_dim"]
    if own:
        rgd, cache, ws = _handle(s)
        rgd.paged_attention(cache, LAYER, s["q"], n, s["new"], ws, s["out"], s["lse"])
        return s["out"], s["lse"]
    pages, lens, new = s["pages"].long(), s["lens"].long(), s["new"].long()
    S, L = len(lens), pages.shape[1] * c["page"]
    ids = pages.clamp(min=0)
    k = s["pool_k"][LAYER][ids].permute(0, 2, 1, 3, 4).reshape(S, hk, L, d).float()
    v = s["pool_v"][LAYER][ids].permute(0, 2, 1, 4, 3).reshape(S, hk, L, d).float()
    pos = torch.arange(L, device="cuda")
    there = (pos < lens[:, None])[:, None, :, None]
    k, v = torch.where(there, k, 0.0), torch.where(there, v, 0.0)
    q = s["q"].float().reshape(S, n, hk, hq // hk, d).permute(0, 2, 3, 1, 4).reshape(S, hk, hq // hk * n, d)
    a = torch.matmul(q, k.transpose(2, 3).contiguous()) / math.sqrt(d)
    end = lens[:, None] - new[:, None] + torch.arange(n, device="cuda") + 1  # positions that token i sees
    seen = (pos < end[:, :, None])[:, None, None].expand(S, hk, hq // hk, n, L).reshape(S, hk, hq // hk * n, L)
    a = torch.where(seen, a, -math.inf)
    top = a.amax(-1, keepdim=True).clamp(min=-3e38)
    e = torch.exp(a - top)
    z = e.sum(-1, keepdim=True)
    o = torch.matmul(e, v) / torch.where(z > 0, z, 1.0)
    lse = (top + torch.log(z)).view(S, hk, hq // hk, n).permute(0, 3, 1, 2).reshape(S * n, hq)
    o = o.view(S, hk, hq // hk, n, d).permute(0, 3, 1, 2, 4).reshape(S * n, hq * d)
    row = (torch.arange(n, device="cuda") < new[:, None]).view(-1, 1)
    s["out"].copy_(torch.where(row, o.to(s["out"].dtype), s["out"]))
    s["lse"].copy_(torch.where(row, lse, s["lse"]))
    return s["out"], s["lse"]


def _append(s, c):
    n = c["n"]
    if own:
        rgd, cache, _ = _handle(s)
        rgd.paged_append(cache, LAYER, s["k"], s["v"], n, s["new"])
    else:
        ps, lens, new = c["page"], s["lens"].long(), s["new"].long()
        i = torch.arange(n, device="cuda")
        pos = lens[:, None] - new[:, None] + i
        row = (i < new[:, None]).view(-1)
        page = s["pages"].long().gather(1, (pos // ps).clamp(max=s["pages"].shape[1] - 1)).view(-1)[row]
        slot = (pos % ps).view(-1)[row]
        s["pool_k"][LAYER][page, :, slot] = s["k"][row]
        s["pool_v"][LAYER][page, :, :, slot] = s["v"][row]
    return _outputs(s)


def _branch(s, c):
    if own:
        rgd, cache, ws = _handle(s)
        rgd.paged_select(cache, s["parent"], s["keep"], ws)
        rgd.paged_reserve(cache, s["grow"], ws)
        return _outputs(s)
    ps, (S, width) = c["page"], s["pages"].shape
    pages, lens, refs = s["pages"].long(), s["lens"].long(), s["refs"].long()
    j = torch.arange(width, device="cuda")
    # the kept positions of each sequence's parent
    parent, keep = s["parent"].long(), s["keep"].long()
    length = torch.where(keep < 0, lens[parent], torch.minimum(keep, lens[parent]))
    had, used = (lens + ps - 1) // ps, (length + ps - 1) // ps
    taken = torch.where(j < used[:, None], pages[parent], torch.where(j < had[:, None], -1, pages))
    refs = refs.scatter_add(0, pages.clamp(min=0).view(-1), -(j < had[:, None]).long().view(-1))
    refs = refs.scatter_add(0, taken.clamp(min=0).view(-1), (j < used[:, None]).long().view(-1))
    # pages for the next tokens: the lowest free ones, in the order of the sequences
    grow = s["grow"].long()
    last = taken.gather(1, (used - 1).clamp(min=0)[:, None])[:, 0].clamp(min=0)
    own_copy = (grow > 0) & (length % ps != 0) & (refs[last] > 1)
    after = (length + grow + ps - 1) // ps
    need = after - used + own_copy.long()
    free = torch.argsort((refs != 0).to(torch.int8), stable=True)
    fits = (need.sum() <= (refs == 0).sum()) & (after <= width).all()
    first = used - own_copy.long()
    fresh = (j >= first[:, None]) & (j < after[:, None]) & fits
    at = (need.cumsum(0) - need)[:, None] + j - first[:, None]
    table = torch.where(fresh, free[at.clamp(0, len(free) - 1)], taken)
    copied = own_copy & fits
    to = table.gather(1, (used - 1).clamp(min=0)[:, None])[:, 0]
    s["pool_k"][:, to[copied]] = s["pool_k"][:, last[copied]]
    s["pool_v"][:, to[copied]] = s["pool_v"][:, last[copied]]
    refs = refs.scatter_add(0, last, -copied.long())
    refs = refs.scatter_add(0, table.clamp(min=0).view(-1), fresh.long().view(-1))
    s["pages"].copy_(table)
    s["lens"].copy_(length + torch.where(fits, grow, 0))
    s["refs"].copy_(refs)
    s["status"].logical_or_(~fits)
    return _outputs(s)


def _compact(s, c):
    s["pages"].copy_(s["before"][0])  # the same scattered state each time
    s["refs"].copy_(s["before"][1])
    if own:
        rgd, cache, ws = _handle(s)
        if "live" not in s:
            s["live"] = torch.zeros(1, dtype=torch.int32, device="cuda")
        rgd.paged_compact(cache, s["live"], ws)
        return {**_outputs(s), "live": s["live"]}
    live = s["refs"] > 0
    n = live.sum()
    ids = torch.arange(len(live), device="cuda")
    move, hole = ids[live & (ids >= n)], ids[~live & (ids < n)]
    s["pool_k"][:, hole] = s["pool_k"][:, move]
    s["pool_v"][:, hole] = s["pool_v"][:, move]
    to = ids.clone()
    to[move] = hole
    s["refs"][hole] = s["refs"][move]
    s["refs"][move] = 0
    used = torch.arange(s["pages"].shape[1], device="cuda") < ((s["lens"].long() + c["page"] - 1) // c["page"])[:, None]
    s["pages"].copy_(torch.where(used, to[s["pages"].long().clamp(min=0)], s["pages"].long()))
    return {**_outputs(s), "live": n.to(torch.int32).view(1)}


def _softmax(z, T, min_p):
    """The truncated distribution of each row in 64 bits; a row without a finite maximum has none (zeros)."""
    z = z.double()
    z = torch.where(torch.isnan(z), -math.inf, z)
    top = z.amax(-1, keepdim=True)
    fine = torch.isfinite(top)
    z = torch.where(fine, z - top, -math.inf)
    if T == 0.0:
        first = torch.zeros_like(z).scatter_(-1, z.argmax(-1, keepdim=True), 1.0)
        return torch.where(fine, first, 0.0), fine[..., 0]
    low = T * math.log(min_p) if min_p > 0 else -math.inf
    w = torch.where(z >= low, torch.exp(z / T), 0.0)
    return w / torch.where(fine, w.sum(-1, keepdim=True), 1.0), fine[..., 0]


def _verify(s, c):
    S, K, V = c["seqs"], c["k"], c["vocab"]
    if own:
        import paper_2607_20791_amd as rgd
        if "ws" not in s:
            s["ws"] = torch.empty(rgd.verify_workspace_bytes(S, K, V), dtype=torch.uint8, device="cuda")
            s["out"] = torch.empty(S, K + 1, dtype=torch.int32, device="cuda")
            s["count"] = torch.empty(S, dtype=torch.int32, device="cuda")
        rgd.verify_drafts(s["target"], s["draft"], s["tokens"], s["n_draft"], c["T"], c["min_p"], s["u"], s["ws"],
                          s["out"], s["count"])
        return s["out"], s["count"]
    T, min_p = float(np.float32(c["T"])), float(np.float32(c["min_p"]))
    p, fine = _softmax(s["target"], T, min_p)
    x = s["tokens"].long()
    inside = (x >= 0) & (x < V)
    at = x.clamp(0, V - 1)[..., None]
    if s["draft"] is None or T == 0.0:
        q = torch.zeros(S, K, V, dtype=torch.float64, device="cuda").scatter_(2, at, inside.double()[..., None])
    else:
        q = _softmax(s["draft"], T, min_p)[0]
    px = torch.where(inside, p[:, :K].gather(2, at)[..., 0], 0.0)
    qx = torch.where(inside, q.gather(2, at)[..., 0], 0.0)
    u = s["u"].double()
    i = torch.arange(K + 1, device="cuda")
    drafted = i[:K] < s["n_draft"].long()[:, None]
    taken = ((u[:, :K] * qx < px) & drafted & fine[:, :K]).long().cumprod(1)
    count = taken.sum(1)
    row = count[:, None, None].expand(S, 1, V)
    r = p.gather(1, row)[:, 0]
    refused = count < s["n_draft"].long().clamp(0, K)
    less = torch.where(refused[:, None], q.gather(1, row.clamp(max=K - 1))[:, 0], 0.0)
    rest = (r - less).clamp(min=0.0)
    rest = torch.where(rest.sum(1, keepdim=True) > 0, rest, r)
    run_sum = rest.cumsum(1)
    token = (run_sum <= u[:, K:] * run_sum[:, -1:]).sum(1).clamp(max=V - 1)
    token = torch.where(fine.gather(1, count[:, None])[:, 0], token, -1)
    out = torch.where(i < count[:, None], torch.nn.functional.pad(x, (0, 1)), -1)
    out = out.scatter(1, count[:, None], token[:, None])
    return out.to(torch.int32), count.to(torch.int32)


# --------------------------------------------------------------------- work --
def work(case):
    c, kind = case, case["kind"]
    if kind == "verify":
        k = _drafts(c)
        rows = int((k + 1).sum()) + (int(k.sum()) if c["draft"] == "logits" and c["T"] > 0 else 0)
        return {"bytes": 4 * rows * c["vocab"] + 4 * c["seqs"] * (3 * c["k"] + 4), "flops": 4 * rows * c["vocab"]}
    block = c["kv_heads"] * c["head_dim"] * 2 * _size(c)  # K and V of one position in one layer
    if kind == "branch":
        P, N, ps = c["prompts"], c["branches"], c["page"]
        forked = sum(int(L) % ps != 0 for L in _spread(P, max(1, c["max_len"] // 4), c["max_len"])) * (N // 2)
        return {"bytes": 2 * forked * c["layers"] * ps * block + 12 * P * (1 + N), "flops": 0}
    if kind == "compact":
        S, ps = c["seqs"], c["page"]
        lens = np.minimum(_spread(S, 20, c["max_len"]), max(1, c["pages"] // 2 // S * ps))
        live = int(_up(lens, ps).sum())
        moved = live * (1 - live / c["pages"])  # expected: the pages lie anywhere
        return {"bytes": 2 * moved * c["layers"] * ps * block + 4 * c["pages"], "flops": 0}
    lens, new = _lengths(c)
    if kind == "append":
        return {"bytes": 2 * int(new.sum()) * block, "flops": 0}
    rows = 2 * int(new.sum()) * c["heads"] * c["head_dim"] * _size(c)
    seen = int((new * lens - new * (new - 1) // 2).sum())
    return {"bytes": int(lens.sum()) * block + rows + 4 * int(new.sum()) * c["heads"],
            "flops": 4 * c["heads"] * c["head_dim"] * seen}


# -------------------------------------------------------------------- exact --
def exact(case, seed):
    c = case
    if c["kind"] == "attention":
        return _exact_attention(prepare(case, seed), c)
    if c["kind"] == "verify" and c["seqs"] * (2 * c["k"] + 1) * c["vocab"] < 1e8:
        return _exact_verify(prepare(case, seed), c)
    return None  # the others place and move values


def _exact_attention(s, c):
    n, hq, hk, d, ps = c["n"], c["heads"], c["kv_heads"], c["head_dim"], c["page"]
    G = hq // hk
    out, lse = s["out"].double(), s["lse"].double()
    q = s["q"].double().view(-1, n, hq, d)
    for b, (L, m) in enumerate(zip(s["lens"].tolist(), s["new"].tolist())):
        ids = s["pages"][b, :_up(L, ps)].long()
        keys = s["pool_k"][LAYER, ids].transpose(0, 1).reshape(hk, -1, d)[:, :L].double()
        vals = s["pool_v"][LAYER, ids].transpose(2, 3).transpose(0, 1).reshape(hk, -1, d)[:, :L].double()
        for i in range(m):
            t = L - m + i + 1
            for h in range(hk):
                a = (q[b, i, h * G:(h + 1) * G] @ keys[h, :t].T) * d ** -0.5
                l = torch.logsumexp(a, 1)
                o = torch.exp(a - l[:, None]) @ vals[h, :t]
                lse[b * n + i, h * G:(h + 1) * G] = l
                out[b * n + i, h * G * d:(h + 1) * G * d] = o.reshape(-1)
    return out, lse


def _exact_verify(s, c):
    S, K, V, T = c["seqs"], c["k"], c["vocab"], float(np.float32(c["T"]))
    floor = float(np.float32(c["min_p"]))

    def probs(z):
        z = z.astype(np.float64)
        if T == 0.0:
            return np.eye(1, V, int(np.argmax(z)))[0]
        e = np.exp((z - z.max()) / T)
        e[z - z.max() < (T * np.log(floor) if floor > 0 else -np.inf)] = 0.0
        return e / math.fsum(e)

    target, tokens, u = s["target"].cpu().numpy(), s["tokens"].cpu().numpy(), s["u"].cpu().numpy().astype(np.float64)
    draft = s["draft"].cpu().numpy() if s["draft"] is not None and T > 0 else None
    out, count = np.full((S, K + 1), -1, np.int32), np.zeros(S, np.int32)
    for b, k in enumerate(s["n_draft"].tolist()):
        for i in range(k + 1):
            rest = p = probs(target[b, i])
            if i < k:
                x = tokens[b, i]
                q = np.eye(1, V, x)[0] if draft is None else probs(draft[b, i])
                if u[b, i] * q[x] < p[x]:
                    out[b, i] = x
                    count[b] += 1
                    continue
                rest = np.maximum(p - q, 0.0)
            total = np.cumsum(rest)
            out[b, i] = np.searchsorted(total, u[b, K] * total[-1], side="right")
            break
    return out, count
