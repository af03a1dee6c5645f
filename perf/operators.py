"""Workloads of the verification step's attention operators: rotary append, attention of drafted trees over a paged
cache, attention weight per cached slot, and eviction from the cache.

One target model verifies drafts of many samples.  Per layer of that model a step takes the projections of the drafted
tokens, rotates queries and keys to their positions and writes keys and values into the paged cache (rope_append),
attends from every drafted token to the cache and to its own ancestors among the drafts (tree_attention), adds up what
attention every cached slot received (cache_weights) and, when the cache is over its budget, keeps the slots that
received most (cache_evict).  A case names one of the four and its sizes; `run` is one call of it."""
import math

import numpy as np
import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16}


# --------------------------------------------------------------------------------------------------------------------
# cases
# --------------------------------------------------------------------------------------------------------------------
def _rope(name, B, tokens, ctx, Hq, Hk, D, rot, layout, scaling, dtype, page):
    return {"name": name, "op": "rope_append", "B": B, "tokens": tokens, "ctx": ctx, "Hq": Hq, "Hk": Hk, "D": D, "rot": rot,
            "layout": layout, "scaling": scaling, "dtype": dtype, "page": page}


def _attn(name, op, B, tree, tokens, ctx, Hq, Hk, D, dtype, page):
    return {"name": name, "op": op, "B": B, "tree": tree, "tokens": tokens, "ctx": ctx, "Hq": Hq, "Hk": Hk, "D": D,
            "dtype": dtype, "page": page}


def _evict(name, B, length, budget, recent, sinks, Hk, D, dtype, page):
    return {"name": name, "op": "cache_evict", "B": B, "len": length, "budget": budget, "recent": recent, "sinks": sinks,
            "Hk": Hk, "D": D, "dtype": dtype, "page": page}


def listed():
    return [
        # the target takes a sample over and writes one token at a time
        _rope("rope one token", 1, 1, 512, 32, 8, 128, 128, "half", "none", "bf16", 16),
        # ragged draft trees, part of the head rotated, interleaved pairs, frequencies rescaled by bands
        _rope("rope 23 trees", 23, 77, 1024, 28, 4, 128, 64, "interleaved", "bands", "fp16", 16),
        # 32 samples' drafts of 500 tokens each, cache positions stretched for a long context
        _rope("rope 32 x 500", 32, 500, 8192, 40, 8, 128, 128, "half", "ramp", "bf16", 64),
        # one token over a draft budget's cache: the latency of a call
        _attn("attend one token", "tree_attention", 1, "chain", 1, 499, 32, 8, 128, "bf16", 16),
        # sixteen samples, each with a small draft tree over its own ragged cache
        _attn("attend 16 trees", "tree_attention", 16, "tree", 24, 2500, 40, 8, 128, "bf16", 16),
        # few drafted tokens over a long reasoning trace: reading the cache is what it costs
        _attn("attend long cache", "tree_attention", 4, "tree", 13, 131071, 32, 8, 128, "fp16", 64),
        # eight drafts of 500 tokens each that share one prompt in the cache
        _attn("attend 8 drafts of 500", "tree_attention", 1, "fan8", 4000, 1013, 40, 8, 128, "bf16", 32),
        # the last quarter of a budget of 8192 tokens, read in again by the target
        _attn("attend chunk of 2048", "tree_attention", 2, "chain", 2048, 6144, 64, 8, 128, "bf16", 128),
        # weights after a step of one token for eight samples
        _attn("weights one token", "cache_weights", 8, "chain", 1, 2000, 32, 8, 128, "bf16", 16),
        # weights of the slots of a shared prompt and of its drafts
        _attn("weights 8 drafts of 500", "cache_weights", 1, "fan8", 4000, 1013, 40, 8, 128, "bf16", 32),
        # a sample's cache of a turn cut back from 700 to 500 slots
        _evict("evict 700 to 500", 4, 700, 500, 64, 4, 8, 128, "bf16", 16),
        # long caches cut back to a budget of 8192
        _evict("evict 32000 to 8192", 8, 32000, 8192, 512, 4, 8, 128, "bf16", 64),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _not_odd_size(n):
    """3072 is left out of every size."""
    return n + 1 if n == 3072 else n


def draw(rng):
    op = rng.choice(["rope_append", "tree_attention", "tree_attention", "cache_weights", "cache_evict"])
    Hq, Hk = rng.choice([(32, 8), (28, 4), (40, 8), (64, 8), (16, 16), (12, 1), (24, 8), (14, 2)])
    D = rng.choice([128, 128, 64])
    dtype = rng.choice(["bf16", "fp16"])
    page = rng.choice([16, 32, 64, 128])
    if op == "rope_append":
        B = _log_int(rng, 1, 32)
        return {k: v for k, v in _rope("", B, _log_int(rng, 1, 500), _not_odd_size(_log_int(rng, 1, 8192)), Hq, Hk, D,
                                       rng.choice([D, D // 2, D // 4]), rng.choice(["half", "interleaved"]),
                                       rng.choice(["none", "bands", "ramp"]), dtype, page).items() if k != "name"}
    if op == "cache_evict":
        B, length = _log_int(rng, 1, 8), _not_odd_size(_log_int(rng, 100, 32000))
        budget = _not_odd_size(max(8, int(length * rng.uniform(0.2, 0.9))))
        recent = rng.randint(0, budget // 4)
        return {k: v for k, v in _evict("", B, length, budget, recent, rng.randint(0, 4), Hk, D, dtype, page).items() if k != "name"}
    kind = rng.choice(["step", "tree", "fan"])
    if kind == "step":       # one token each, over caches of any length
        B, tree, tokens, ctx = _log_int(rng, 1, 64), "chain", 1, _log_int(rng, 1, 16384)
    elif kind == "tree":     # small trees
        B, tree, tokens, ctx = _log_int(rng, 1, 24), "tree", _log_int(rng, 2, 96), _log_int(rng, 1, 8192)
    else:                    # whole drafts that share their prompt
        B, tokens, ctx = rng.randint(1, 2), _log_int(rng, 200, 2000), _log_int(rng, 1, 2048)
        tree = rng.choice(["chain", "fan4", "fan7"])
    return {k: v for k, v in _attn("", op, B, tree, _not_odd_size(tokens), _not_odd_size(ctx), Hq, Hk, D, dtype, page).items()
            if k != "name"}


# --------------------------------------------------------------------------------------------------------------------
# what a case's batch looks like (host side, from the sizes and the seed)
# --------------------------------------------------------------------------------------------------------------------
def _ragged(most, B):
    """B whole numbers from 60 % of `most` to `most`, the largest among them: the same for a case whatever its seed, so
    that its outputs have one shape."""
    rs = np.random.RandomState([most, B])
    n = rs.randint(max(0, int(0.6 * most)), most + 1, size=B)
    n[rs.randint(B)] = most
    return n.astype(np.int64)


def _parents(rs, tree, T):
    """Parent of each of T drafted tokens, -1 where it hangs on the cache; parents come before their children."""
    if tree == "chain":
        return np.arange(-1, T - 1)
    if tree.startswith("fan"):
        each = -(-T // int(tree[3:]))
        i = np.arange(T)
        return np.where(i % each == 0, -1, i - 1)
    i = np.arange(T)      # a draft tree in level order: about three tokens a level hang on one of the level before
    return np.where(i < 3, -1, np.maximum(i - 3 - rs.randint(0, 3, size=T), 0))


def _preorder(parent):
    """(pre, end, depth): place of each token in the tree's preorder, one past its last descendant's place, its depth.
    Token j is an ancestor of i, or i itself, where pre[j] <= pre[i] < end[j]."""
    T = len(parent)
    size, depth = np.ones(T, np.int64), np.zeros(T, np.int64)
    for i in range(T - 1, -1, -1):
        if parent[i] >= 0:
            size[parent[i]] += size[i]
    pre, nxt, top = np.zeros(T, np.int64), np.zeros(T, np.int64), 0
    for i in range(T):
        p = parent[i]
        if p < 0:
            pre[i], top = top, top + size[i]
        else:
            pre[i], nxt[p], depth[i] = nxt[p], nxt[p] + size[i], depth[p] + 1
        nxt[i] = pre[i] + 1
    return pre, pre + size, depth


def _batch(case, seed):
    rs = np.random.RandomState([seed % (1 << 31), 77])
    B, T = case["B"], case["tokens"]
    tokens, ctx = np.maximum(_ragged(T, B), 1), _ragged(case["ctx"], B)
    tree = case.get("tree", "tree")
    parent = [_parents(rs, tree, int(t)) for t in tokens]
    return rs, tokens, ctx, parent


def _visible(case, seed):
    """(pairs of a token and a slot it sees, tokens, slots) of the whole batch."""
    _, tokens, ctx, parent = _batch(case, seed)
    pairs = 0
    for t, c, p in zip(tokens, ctx, parent):
        pairs += int(t) * int(c) + int((_preorder(p)[2] + 1).sum())
    return pairs, int(tokens.sum()), int((tokens + ctx).sum())


def _dev(x, dtype=torch.int32):
    return torch.from_numpy(np.ascontiguousarray(x)).to("cuda", dtype)


def _pages(rs, need, B, page):
    """Block table [B, most pages] with the pages of all sequences shuffled, and the number of pages."""
    each = -(-need // page)
    total = int(each.sum())
    perm = rs.permutation(total)
    table = np.zeros((B, max(1, int(each.max()))), np.int64)
    at = 0
    for b in range(B):
        table[b, : each[b]] = perm[at : at + each[b]]
        at += int(each[b])
    return table, max(1, total)


def _freqs(case):
    """Rotations per position in radians, in 64 bits, and the factor on cosine and sine."""
    r = case["rot"]
    base, factor, orig = 1000000.0 if case["scaling"] == "none" else 500000.0, 8.0, 8192.0
    f = base ** (-np.arange(0, r, 2, dtype=np.float64) / r)
    if case["scaling"] == "bands":
        low, high = 1.0, 4.0
        turns = orig * f / (2 * math.pi)
        s = np.clip((turns - low) / (high - low), 0.0, 1.0)
        return (1 - s) * f / factor + s * f, 1.0
    if case["scaling"] == "ramp":
        at = lambda n: r * math.log(orig / (n * 2 * math.pi)) / (2 * math.log(base))  # noqa: E731
        lo, hi = max(math.floor(at(32.0)), 0), min(math.ceil(at(1.0)), r - 1)
        ramp = np.clip((np.arange(r // 2) - lo) / max(hi - lo, 1e-3), 0.0, 1.0)
        return f * (1 - ramp) + f / factor * ramp, 0.1 * math.log(factor) + 1.0
    return f, 1.0


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(int(seed) + 1)
    dt, page = DTYPES[case["dtype"]], case["page"]
    randn = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    st = {"op": case["op"], "page": page}
    Hk, D = case["Hk"], case["D"]

    if case["op"] == "cache_evict":
        rs = np.random.RandomState([int(seed) % (1 << 31), 78])
        B, budget = case["B"], case["budget"]
        lens = np.maximum(_ragged(case["len"], B), 1)
        table, n_pages = _pages(rs, lens, B, page)
        keep = np.minimum(lens, budget)
        out_table, n_out = _pages(rs, keep, B, page)
        st["k"], st["v"] = randn(n_pages, page, Hk, D).to(dt), randn(n_pages, page, Hk, D).to(dt)
        st["table"], st["lens"] = _dev(table), _dev(lens)
        # what slots receive is spread over decades; a slot that nobody looked at has exactly zero, and ties happen
        w = torch.exp(2.0 * randn(B, Hk, int(lens.max())) - 3.0)
        w[torch.rand(w.shape, generator=g, device="cuda") < 0.05] = 0.0
        st["weights"] = torch.where(w > 1.0, torch.round(w * 8) / 8, w).contiguous()
        st["out_table"] = _dev(out_table)
        st["k_out"], st["v_out"] = torch.zeros(n_out, page, Hk, D, dtype=dt, device="cuda"), torch.zeros(n_out, page, Hk, D, dtype=dt, device="cuda")
        st["kept"] = torch.empty(B, Hk, budget, dtype=torch.int32, device="cuda")
        st["counts"] = torch.empty(B, dtype=torch.int32, device="cuda")
        st["weights_out"] = torch.empty(B, Hk, budget, device="cuda")
        st.update(budget=budget, recent=case["recent"], sinks=case["sinks"])
        if own:
            from paper_2509_15148_b200 import binding
            st["cache"], st["out_cache"] = binding.PagedCache(st["k"], st["v"], st["table"]), binding.PagedCache(st["k_out"], st["v_out"], st["out_table"])
        return st

    rs, tokens, ctx, parent = _batch(case, int(seed))
    B, Hq = case["B"], case["Hq"]
    M = int(tokens.sum())
    table, n_pages = _pages(rs, tokens + ctx, B, page)
    cu = np.concatenate([[0], np.cumsum(tokens)])
    st["table"], st["ctx"], st["cu"] = _dev(table), _dev(ctx), _dev(cu)
    st["max_tokens"], st["max_len"] = int(tokens.max()), int((tokens + ctx).max())
    trees = [_preorder(p) for p in parent]
    pre, end, depth = (np.concatenate([t[k] for t in trees]) for k in range(3))

    if case["op"] == "rope_append":
        # queries, keys and values as one projection leaves them: views of one row per token
        qkv = randn(M, (Hq + 2 * Hk) * D).to(dt)
        st["q"], st["k_new"], st["v_new"] = (t.unflatten(1, (-1, D)) for t in qkv.split([Hq * D, Hk * D, Hk * D], dim=1))
        st["k"], st["v"] = randn(n_pages, page, Hk, D).to(dt), randn(n_pages, page, Hk, D).to(dt)
        st["positions"] = _dev(np.repeat(ctx, tokens) + depth)
        f, st["mscale"] = _freqs(case)
        st["freqs"] = torch.from_numpy(f).cuda()
        st["interleaved"] = case["layout"] == "interleaved"
        st["q_out"] = torch.empty(M, Hq, D, dtype=dt, device="cuda")
        if own:
            from paper_2509_15148_b200 import binding
            st["cache"] = binding.PagedCache(st["k"], st["v"], st["table"])
        return st

    # Queries lean towards a direction in which the first few slots of a cache are strong, as trained models' do.
    u = torch.nn.functional.normalize(randn(Hk, D), dim=-1)
    G = Hq // Hk
    st["q"] = (randn(M, Hq, D) + 4.0 * u.repeat_interleave(G, 0)).to(dt)
    k = randn(n_pages, page, Hk, D)
    first = _dev(table[:, 0], torch.int64)
    k[first, : min(4, page)] += 10.0 * u
    st["k"], st["v"] = k.to(dt), randn(n_pages, page, Hk, D).to(dt)
    del k
    chain = case["tree"] == "chain"
    st["pre"], st["end"] = (None, None) if chain else (_dev(pre), _dev(end))
    st["scale"] = 1.0 / math.sqrt(D)
    if case["op"] == "cache_weights":
        st["lse"] = _attend(st, want_out=False)[1]
        st["weights"] = torch.rand(B, Hk, st["max_len"], generator=g, device="cuda")
        st["weights_out"] = torch.zeros_like(st["weights"])
    else:
        st["out"], st["lse"] = torch.empty(M, Hq, D, dtype=dt, device="cuda"), torch.empty(M, Hq, device="cuda")
    if own:
        from paper_2509_15148_b200 import binding
        st["cache"] = binding.PagedCache(st["k"], st["v"], st["table"])
        if case["op"] == "tree_attention":
            n = binding.tree_attention_workspace_bytes(B, M, Hq, Hk, D, st["max_tokens"], st["max_len"])
            st["workspace"] = torch.empty(n, dtype=torch.uint8, device="cuda")
    return st


# --------------------------------------------------------------------------------------------------------------------
# one pass
# --------------------------------------------------------------------------------------------------------------------
def run(st):
    if own:
        return _run_own(st)
    if st["op"] == "rope_append":
        return _rope_append(st)
    if st["op"] == "tree_attention":
        out, lse = _attend(st)
        return {"out": out, "lse": lse}
    if st["op"] == "cache_weights":
        return {"weights": _weights(st)}
    return _evict_plain(st)


def _run_own(st):
    from paper_2509_15148_b200 import binding
    if st["op"] == "rope_append":
        binding.rope_append(st["q"], st["k_new"], st["v_new"], st["positions"], st["freqs"], st["cache"], st["ctx"], st["cu"],
                            st["max_tokens"], st["q_out"], interleaved=st["interleaved"], mscale=st["mscale"])
        return {"q": st["q_out"], "k": st["k"], "v": st["v"]}
    if st["op"] == "tree_attention":
        binding.tree_attention(st["q"], st["cache"], st["ctx"], st["cu"], st["pre"], st["end"], st["max_tokens"], st["max_len"],
                               st["scale"], st["out"], st["lse"], st["workspace"])
        return {"out": st["out"], "lse": st["lse"]}
    if st["op"] == "cache_weights":
        binding.cache_weights(st["q"], st["cache"], st["lse"], st["ctx"], st["cu"], st["pre"], st["end"], st["max_tokens"],
                              st["max_len"], st["scale"], st["weights"], st["weights_out"])
        return {"weights": st["weights_out"]}
    binding.cache_select(st["weights"], st["lens"], st["budget"], st["sinks"], st["recent"], st["kept"], st["counts"])
    binding.cache_gather(st["cache"], st["kept"], st["counts"], st["out_cache"], st["weights"], st["weights_out"])
    return {"kept": st["kept"], "counts": st["counts"], "k": st["k_out"], "v": st["v_out"], "weights": st["weights_out"]}


def _where(st):
    """(sequence, place in it) of every token."""
    cu = st["cu"].long()
    i = torch.arange(st["q"].shape[0], device="cuda")
    b = torch.searchsorted(cu, i, right=True) - 1
    return b, i - cu[b]


def _rotate(x, c, s, half, interleaved):
    x = x.float()
    y = x.clone()
    if interleaved:
        a, b = x[..., 0 : 2 * half : 2], x[..., 1 : 2 * half : 2]
        y[..., 0 : 2 * half : 2], y[..., 1 : 2 * half : 2] = a * c - b * s, b * c + a * s
    else:
        a, b = x[..., :half], x[..., half : 2 * half]
        y[..., :half], y[..., half : 2 * half] = a * c - b * s, b * c + a * s
    return y


def _rope_append(st):
    b, t = _where(st)
    angle = st["positions"].float()[:, None] * st["freqs"].float()
    c, s = ((f(angle) * st["mscale"])[:, None] for f in (torch.cos, torch.sin))
    half = st["freqs"].numel()
    q = _rotate(st["q"], c, s, half, st["interleaved"]).to(st["q"].dtype)
    k = _rotate(st["k_new"], c, s, half, st["interleaved"]).to(st["k"].dtype)
    slot = st["ctx"].long()[b] + t
    page = st["table"].long()[b, slot // st["page"]]
    st["k"][page, slot % st["page"]] = k
    st["v"][page, slot % st["page"]] = st["v_new"]
    return {"q": q, "k": st["k"], "v": st["v"]}


def _scores(st):
    """Scaled scores [B, Hk, tokens * G, slots] with -inf where a token does not see a slot, and what belongs to them."""
    b, t = _where(st)
    M, Hq, D = st["q"].shape
    B, T, S = st["ctx"].numel(), st["max_tokens"], st["max_len"]
    Hk = st["k"].shape[2]
    G = Hq // Hk
    slot = torch.arange(S, device="cuda")
    cu, ctx = st["cu"].long(), st["ctx"].long()
    n = cu[1:] - cu[:-1]
    live = slot[None] < (ctx + n)[:, None]                                   # [B, S]
    page = torch.where(live, st["table"].long()[:, slot.clamp(max=st["table"].shape[1] * st["page"] - 1) // st["page"]], 0)
    off = (slot % st["page"])[None].expand(B, S)
    q = torch.zeros(B, T, Hq, D, device="cuda")
    q[b, t] = st["q"].float()
    q = q.unflatten(2, (Hk, G)).permute(0, 2, 1, 3, 4).reshape(B, Hk, T * G, D)
    k = st["k"][page, off].float().permute(0, 2, 3, 1)                       # [B, Hk, D, S]
    s = torch.matmul(q, k).mul_(st["scale"])
    # the tree: a drafted slot is seen by itself and its descendants
    i = torch.arange(M, device="cuda") - cu[b]
    pre_flat = st["pre"].long() if st["pre"] is not None else i
    end_flat = st["end"].long() if st["pre"] is not None else n[b]
    pre, lo, hi = (torch.full(x, v, device="cuda") for x, v in (((B, T), -1), ((B, S), 1 << 30), ((B, S), 0)))
    pre[b, t] = pre_flat
    lo[b, ctx[b] + t], hi[b, ctx[b] + t] = pre_flat, end_flat
    old = slot[None] < ctx[:, None]
    lo, hi = torch.where(old, 0, lo), torch.where(old, 1 << 30, hi)
    see = (lo[:, None] <= pre[:, :, None]) & (pre[:, :, None] < hi[:, None]) & live[:, None]   # [B, T, S]
    s.view(B, Hk, T, G, S).masked_fill_(~see[:, None, :, None], float("-inf"))
    return s, b, t, page, off, live, (B, Hk, T, G, S, D)


def _rows(x, b, t, shape):
    """[B, Hk, T * G, ...] -> [tokens, Hq, ...]"""
    B, Hk, T, G, S, D = shape
    return x.view(B, Hk, T, G, -1)[b, :, t].flatten(1, 2)


def _attend(st, want_out=True):
    s, b, t, page, off, live, shape = _scores(st)
    m = s.amax(-1, keepdim=True)
    m = torch.where(m == float("-inf"), 0.0, m)
    p = s.sub_(m).exp_()
    l = p.sum(-1, keepdim=True)
    lse = _rows(m + torch.log(l), b, t, shape).squeeze(-1).contiguous()
    if not want_out:
        return None, lse
    v = torch.where(live[:, :, None, None], st["v"][page, off].float(), 0.0).permute(0, 2, 1, 3)
    o = torch.matmul(p, v) / torch.where(l == 0, 1.0, l)
    return _rows(o, b, t, shape).to(st["q"].dtype), lse


def _weights(st):
    s, b, t, page, off, live, shape = _scores(st)
    B, Hk, T, G, S, D = shape
    lse = torch.full((B, T, Hk, G), float("inf"), device="cuda")
    lse[b, t] = st["lse"].view(-1, Hk, G)
    p = s.view(B, Hk, T, G, S).sub_(lse.permute(0, 2, 1, 3)[..., None]).exp_()
    return torch.where(live[:, None], st["weights"] + p.sum((2, 3)), 0.0)


def _evict_plain(st):
    w, lens, budget = st["weights"], st["lens"].long(), st["budget"]
    B, Hk, S = w.shape
    slot = torch.arange(S, device="cuda")
    live = slot[None] < lens[:, None]
    must = live & ((slot[None] < st["sinks"]) | (slot[None] >= (lens - st["recent"])[:, None]))
    key = torch.where(live[:, None], torch.where(must[:, None], float("inf"), w), float("-inf"))
    order = torch.sort(key, dim=-1, descending=True, stable=True)[1][..., :budget]
    counts = torch.clamp(lens, max=budget)
    if S < budget:
        order = torch.nn.functional.pad(order, (0, budget - S))
    place = torch.arange(budget, device="cuda")
    has = (place[None] < counts[:, None])[:, None].expand(B, Hk, budget)
    kept = torch.sort(torch.where(has, order, 1 << 30), dim=-1)[0]
    at = torch.where(has, kept, 0)
    b = torch.arange(B, device="cuda")[:, None, None]
    h = torch.arange(Hk, device="cuda")[None, :, None]
    page, off = st["table"].long()[b, at // st["page"]], at % st["page"]
    to = place[None].expand(B, budget)
    ok = place[None] < counts[:, None]
    to_page = st["out_table"].long()[b[..., 0], (to // st["page"]).clamp(max=st["out_table"].shape[1] - 1)]
    for_k, for_v = (st[x][page, off, h].permute(0, 2, 1, 3) for x in ("k", "v"))      # [B, budget, Hk, D]
    st["k_out"][to_page[ok], (to % st["page"])[ok]] = for_k[ok]
    st["v_out"][to_page[ok], (to % st["page"])[ok]] = for_v[ok]
    return {"kept": torch.where(has, kept, -1).int(), "counts": counts.int(), "k": st["k_out"], "v": st["v_out"],
            "weights": torch.where(has, torch.gather(w, 2, at), 0.0)}


# --------------------------------------------------------------------------------------------------------------------
# the work that no implementation can do without
# --------------------------------------------------------------------------------------------------------------------
def work(case):
    Hk, D = case["Hk"], case["D"]
    if case["op"] == "cache_evict":
        lens = np.maximum(_ragged(case["len"], case["B"]), 1)
        L, K = int(lens.sum()), int(np.minimum(lens, case["budget"]).sum())
        return {"bytes": Hk * (4 * L + K * (2 * 2 * 2 * D + 8 + 4)), "flops": Hk * L}
    if case["op"] == "rope_append":
        _, tokens, _, _ = _batch(case, 1)
        M = int(tokens.sum())
        return {"bytes": M * (2 * 2 * D * (case["Hq"] + 2 * Hk) + 4), "flops": 3 * M * case["rot"] * (case["Hq"] + Hk)}
    pairs, M, slots = _visible(case, 1)
    Hq = case["Hq"]
    if case["op"] == "cache_weights":
        return {"bytes": 2 * D * (M * Hq + slots * Hk) + 4 * M * Hq + 8 * slots * Hk, "flops": 2 * D * Hq * pairs}
    return {"bytes": 2 * D * (2 * M * Hq + 2 * slots * Hk) + 4 * M * Hq, "flops": 4 * D * Hq * pairs}


# --------------------------------------------------------------------------------------------------------------------
# the definitions in 64 bits, one sequence and head at a time
# --------------------------------------------------------------------------------------------------------------------
def exact(case, seed):
    st = prepare(case, seed)
    if case["op"] == "rope_append":
        return _exact_rope(case, seed, st)
    if case["op"] == "cache_evict":
        return _exact_evict(case, st)
    return _exact_attention(case, seed, st)


def _exact_rope(case, seed, st):
    _, tokens, ctx, parent = _batch(case, int(seed))
    page, r = case["page"], case["rot"]
    angle = st["positions"].double()[:, None] * st["freqs"]
    turn = torch.polar(torch.full_like(angle, float(st["mscale"])), angle)[:, None]      # one complex number per pair

    def rotated(x):
        x = x.double()
        z = x[..., :r].unflatten(-1, (r // 2, 2)) if case["layout"] == "interleaved" else x[..., :r].unflatten(-1, (2, r // 2)).transpose(-1, -2)
        z = torch.view_as_real(torch.view_as_complex(z.contiguous()) * turn)
        z = z if case["layout"] == "interleaved" else z.transpose(-1, -2)
        return torch.cat([z.flatten(-2), x[..., r:]], dim=-1)

    q, k = rotated(st["q"]), rotated(st["k_new"])
    kc, vc = st["k"].double(), st["v"].double()
    table, at = st["table"].tolist(), 0
    for b in range(case["B"]):
        n, c = int(tokens[b]), int(ctx[b])
        slots = torch.arange(c, c + n)
        pages = torch.tensor([table[b][int(x) // page] for x in slots], device="cuda")
        offs = (slots % page).cuda()
        kc[pages, offs], vc[pages, offs] = k[at : at + n], st["v_new"][at : at + n].double()
        at += n
    return {"q": q, "k": kc, "v": vc}


def _sees(parent, ctx):
    """Truth values [tokens, slots]: the cache, and a token's line of parents."""
    T = len(parent)
    see = np.zeros((T, T), bool)
    for i in range(T):
        if parent[i] >= 0:
            see[i, : parent[i] + 1] = see[parent[i], : parent[i] + 1]
        see[i, i] = True
    return torch.from_numpy(np.concatenate([np.ones((T, ctx), bool), see], axis=1)).cuda()


def _exact_attention(case, seed, st):
    _, tokens, ctx, parent = _batch(case, int(seed))
    Hq, Hk, D, page = case["Hq"], case["Hk"], case["D"], case["page"]
    G = Hq // Hk
    weights = case["op"] == "cache_weights"
    M = st["q"].shape[0]
    if weights:
        acc = torch.zeros(st["weights"].shape, dtype=torch.float64, device="cuda")
    else:
        out, lse = torch.zeros(M, Hq, D, dtype=torch.float64, device="cuda"), torch.zeros(M, Hq, dtype=torch.float64, device="cuda")
    at = 0
    for b in range(case["B"]):
        n, S = int(tokens[b]), int(tokens[b] + ctx[b])
        see = _sees(parent[b], int(ctx[b]))
        pages = st["table"][b, : -(-S // page)].long()
        for h in range(Hk):
            k = st["k"][pages, :, h].flatten(0, 1)[:S].double()
            v = st["v"][pages, :, h].flatten(0, 1)[:S].double()
            for g in range(h * G, (h + 1) * G):
                s = (st["q"][at : at + n, g].double() @ k.T) * st["scale"]
                s[~see] = float("-inf")
                if weights:
                    w = torch.exp(s - st["lse"][at : at + n, g].double()[:, None]).sum(0)
                    acc[b, h, :S] += w
                else:
                    lse[at : at + n, g] = torch.logsumexp(s, -1)
                    out[at : at + n, g] = torch.softmax(s, -1) @ v
            if weights:
                acc[b, h, :S] += st["weights"][b, h, :S].double()
        at += n
    return {"weights": acc} if weights else {"out": out, "lse": lse}


def _exact_evict(case, st):
    B, Hk, budget, page = case["B"], case["Hk"], case["budget"], case["page"]
    w = st["weights"].cpu().numpy()
    k_out, v_out = st["k_out"].double(), st["v_out"].double()
    w_out = torch.zeros(B, Hk, budget, dtype=torch.float64)
    table, out_table = st["table"].cpu().numpy(), st["out_table"].cpu().numpy()
    for b, n in enumerate(st["lens"].tolist()):
        for h in range(Hk):
            i = np.arange(n)
            must = (i < case["sinks"]) | (i >= n - case["recent"])
            best = np.lexsort((i, -w[b, h, :n].astype(np.float64), ~must))[:budget]     # the must first, then the largest, then the lowest
            best = np.sort(best)
            c = np.arange(len(best))
            src = [torch.from_numpy(x.astype(np.int64)).cuda() for x in (table[b, best // page], best % page)]
            dst = [torch.from_numpy(x.astype(np.int64)).cuda() for x in (out_table[b, c // page], c % page)]
            k_out[dst[0], dst[1], h] = st["k"][src[0], src[1], h].double()
            v_out[dst[0], dst[1], h] = st["v"][src[0], src[1], h].double()
            w_out[b, h, : len(best)] = torch.from_numpy(w[b, h, best].astype(np.float64))
    return {"kept": None, "counts": None, "k": k_out, "v": v_out, "weights": w_out.cuda()}
