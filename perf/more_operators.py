"""Workloads of further attention operators of a verification step: queries and keys normed per head and rotated on their
way into the paged cache, attention through a sliding window with sinks, and a cache that holds keys and values in 4 bits.

A target model that norms its queries and keys does so in every layer before the rotation (norm_rope_append).  Layers with a
window attend to the last `window` tokens of a draft's own line and to the first few (window_attention).  A cache in 4 bits
takes the drafted tokens' keys and values (packed_append, read back by packed_read) and is attended to as it is
(packed_attention, with or without a window).  A case names one of the four and its sizes; `run` is one pass of it."""
import math

import numpy as np
import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16}
EPS = 1e-6


# --------------------------------------------------------------------------------------------------------------------
# cases
# --------------------------------------------------------------------------------------------------------------------
def _rope(name, B, tokens, ctx, Hq, Hk, D, rot, layout, scaling, dtype, page):
    return {"name": name, "op": "norm_rope_append", "B": B, "tree": "tree", "tokens": tokens, "ctx": ctx, "Hq": Hq, "Hk": Hk, "D": D,
            "rot": rot, "layout": layout, "scaling": scaling, "dtype": dtype, "page": page}


def _append(name, B, tree, tokens, ctx, Hk, D, dtype, page):
    return {"name": name, "op": "packed_append", "B": B, "tree": tree, "tokens": tokens, "ctx": ctx, "Hq": Hk, "Hk": Hk, "D": D,
            "dtype": dtype, "page": page}


def _attn(name, op, B, tree, tokens, ctx, Hq, Hk, D, window, sinks, dtype, page):
    return {"name": name, "op": op, "B": B, "tree": tree, "tokens": tokens, "ctx": ctx, "Hq": Hq, "Hk": Hk, "D": D,
            "window": window, "sinks": sinks, "dtype": dtype, "page": page}


def listed():
    return [
        # the target takes a sample over and writes one token at a time
        _rope("norm rope one token", 1, 1, 512, 32, 8, 128, 128, "half", "none", "bf16", 16),
        # ragged draft trees, half of each head rotated, interleaved pairs, frequencies rescaled by bands
        _rope("norm rope 23 trees", 23, 77, 1024, 28, 4, 128, 64, "interleaved", "bands", "fp16", 16),
        # 32 samples' drafts of 500 tokens each
        _rope("norm rope 32 x 500", 32, 500, 8192, 40, 8, 128, 128, "half", "none", "bf16", 64),
        # one token of eight samples over long caches of which a layer sees 1024 slots
        _attn("window one token", "window_attention", 8, "chain", 1, 8192, 32, 8, 128, 1024, 4, "bf16", 16),
        # sixteen samples, each with a small draft tree; the window's edge lies at another slot for every token
        _attn("window 16 trees", "window_attention", 16, "tree", 24, 5000, 40, 8, 128, 500, 4, "fp16", 16),
        # the last quarter of a budget of 8192 tokens, read in again by the target
        _attn("window chunk of 2048", "window_attention", 2, "chain", 2048, 6144, 64, 8, 128, 1024, 4, "bf16", 128),
        # a step's draft trees go into the cache
        _append("packed append 8 trees", 8, "tree", 24, 500, 8, 128, "bf16", 16),
        # 32 samples' drafts of 500 tokens each
        _append("packed append 32 x 500", 32, "chain", 500, 1, 8, 128, "bf16", 64),
        # one token of eight samples: the latency of a call
        _attn("packed one token", "packed_attention", 8, "chain", 1, 2000, 32, 8, 128, 0, 0, "bf16", 16),
        # sixteen samples, each with a small draft tree over its own ragged cache
        _attn("packed 16 trees", "packed_attention", 16, "tree", 24, 2500, 40, 8, 128, 0, 0, "bf16", 16),
        # few drafted tokens over a long reasoning trace: reading the cache is what it costs
        _attn("packed long cache", "packed_attention", 4, "tree", 13, 131071, 32, 8, 128, 0, 0, "fp16", 64),
        # eight drafts of 500 tokens each that share one prompt in the cache
        _attn("packed 8 drafts of 500", "packed_attention", 1, "fan8", 4000, 1013, 40, 8, 128, 0, 0, "bf16", 32),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["norm_rope_append", "window_attention", "packed_append", "packed_attention", "packed_attention"])
    Hq, Hk = rng.choice([(32, 8), (28, 4), (40, 8), (64, 8), (16, 16), (12, 1), (24, 8), (14, 2)])
    D = rng.choice([128, 128, 64])
    dtype = rng.choice(["bf16", "fp16"])
    page = rng.choice([16, 32, 64, 128])
    if op == "norm_rope_append":
        case = _rope("", _log_int(rng, 1, 32), _log_int(rng, 1, 500), _log_int(rng, 1, 8192), Hq, Hk, D, rng.choice([D, D // 2, D // 4]),
                     rng.choice(["half", "interleaved"]), rng.choice(["none", "bands"]), dtype, page)
    elif op == "packed_append":
        case = _append("", _log_int(rng, 1, 32), rng.choice(["tree", "chain"]), _log_int(rng, 1, 500), _log_int(rng, 1, 500), min(Hk, 8), D, dtype, page)
    else:
        kind = rng.choice(["step", "tree", "fan"])
        if kind == "step":       # one token each, over caches of any length
            B, tree, tokens, ctx = _log_int(rng, 1, 16), "chain", 1, _log_int(rng, 1, 16384)
        elif kind == "tree":     # small trees
            B, tree, tokens, ctx = _log_int(rng, 1, 24), "tree", _log_int(rng, 2, 96), _log_int(rng, 1, 8192)
        else:                    # whole drafts that share their prompt
            B, tokens, ctx = rng.randint(1, 2), _log_int(rng, 200, 2000), _log_int(rng, 1, 2048)
            tree = rng.choice(["chain", "fan4", "fan7"])
        window = _log_int(rng, 1, 4096) if op == "window_attention" else rng.choice([0, 0, _log_int(rng, 64, 4096)])
        case = _attn("", op, B, tree, tokens, ctx, Hq, Hk, D, window, rng.randint(0, 8) if window else 0, dtype, page)
    del case["name"]
    return case


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
    i = np.arange(T)
    if tree == "chain":
        return i - 1
    if tree.startswith("fan"):
        each = -(-T // int(tree[3:]))
        return np.where(i % each == 0, -1, i - 1)
    # a draft tree in level order: about three tokens a level hang on one of the level before
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
    tokens, ctx = np.maximum(_ragged(case["tokens"], case["B"]), 1), _ragged(case["ctx"], case["B"])
    parent = [_parents(rs, case["tree"], int(t)) for t in tokens]
    return rs, tokens, ctx, parent


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
    """Rotations per position in radians, in 64 bits."""
    r = case["rot"]
    base, factor, orig = 1000000.0 if case["scaling"] == "none" else 500000.0, 8.0, 8192.0
    f = base ** (-np.arange(0, r, 2, dtype=np.float64) / r)
    if case["scaling"] == "bands":
        s = np.clip((orig * f / (2 * math.pi) - 1.0) / 3.0, 0.0, 1.0)
        return (1 - s) * f / factor + s * f
    return f


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(int(seed) + 1)
    dt, page = DTYPES[case["dtype"]], case["page"]
    randn = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    Hq, Hk, D, B = case["Hq"], case["Hk"], case["D"], case["B"]
    rs, tokens, ctx, parent = _batch(case, int(seed))
    M = int(tokens.sum())
    table, n_pages = _pages(rs, tokens + ctx, B, page)
    st = {"op": case["op"], "page": page, "table": _dev(table), "ctx": _dev(ctx), "cu": _dev(np.concatenate([[0], np.cumsum(tokens)])),
          "max_tokens": int(tokens.max()), "max_len": int((tokens + ctx).max())}
    trees = [_preorder(p) for p in parent]
    pre, end, depth = (np.concatenate([t[k] for t in trees]) for k in range(3))

    if case["op"] == "norm_rope_append":
        # queries, keys and values as one projection leaves them: views of one row per token
        qkv = (3.0 * randn(M, (Hq + 2 * Hk) * D)).to(dt)
        st["q"], st["k_new"], st["v_new"] = (t.unflatten(1, (-1, D)) for t in qkv.split([Hq * D, Hk * D, Hk * D], dim=1))
        st["q_gain"], st["k_gain"] = (1.0 + 0.3 * randn(D)).to(dt), (1.0 + 0.3 * randn(D)).to(dt)
        st["k"], st["v"] = randn(n_pages, page, Hk, D).to(dt), randn(n_pages, page, Hk, D).to(dt)
        st["positions"] = _dev(np.repeat(ctx, tokens) + depth)
        st["freqs"] = torch.from_numpy(_freqs(case)).cuda()
        st["interleaved"] = case["layout"] == "interleaved"
        st["q_out"] = torch.empty(M, Hq, D, dtype=dt, device="cuda")
        if own:
            from paper_2509_15148_b200 import binding
            st["cache"] = binding.PagedCache(st["k"], st["v"], st["table"])
        return st

    if case["op"] == "packed_append":
        # Keys have some channels that are strong in every token, as trained models' do.
        strong = torch.where(torch.rand(Hk, D, generator=g, device="cuda") < 0.03, 4.0, 1.0)
        st["k_new"], st["v_new"] = (randn(M, Hk, D) * strong).to(dt), randn(M, Hk, D).to(dt)
        cached = [(randn(n_pages, page, Hk, D) * s).to(dt) for s in (strong, torch.ones_like(strong))]
        st["kp"], st["vp"] = (_pack(x) for x in cached)
        st["lens"] = _dev(tokens + ctx)
        st["k"], st["v"] = (torch.zeros(n_pages, page, Hk, D, dtype=dt, device="cuda") for _ in range(2))
        if own:
            from paper_2509_15148_b200 import binding
            st["packed"] = binding.PackedCache(st["kp"], st["vp"], st["table"], page, D)
            st["cache"] = binding.PagedCache(st["k"], st["v"], st["table"])
        return st

    # Queries lean towards a direction in which the first few slots of a cache are strong, as trained models' do.
    u = torch.nn.functional.normalize(randn(Hk, D), dim=-1)
    st["q"] = (randn(M, Hq, D) + 4.0 * u.repeat_interleave(Hq // Hk, 0)).to(dt)
    k = randn(n_pages, page, Hk, D)
    k[_dev(table[:, 0], torch.int64), : min(4, page)] += 10.0 * u
    v = randn(n_pages, page, Hk, D)
    if case["op"] == "window_attention":
        st["k"], st["v"] = k.to(dt), v.to(dt)
    else:
        st["kp"], st["vp"] = _pack(k.to(dt)), _pack(v.to(dt))
    del k, v
    st["pre"], st["end"], st["depth"] = (None,) * 3 if case["tree"] == "chain" else (_dev(pre), _dev(end), _dev(depth))
    st["window"], st["sinks"], st["Hk"] = case["window"], case["sinks"], Hk
    st["scale"] = 1.0 / math.sqrt(D)
    st["out"], st["lse"] = torch.empty(M, Hq, D, dtype=dt, device="cuda"), torch.empty(M, Hq, device="cuda")
    if own:
        from paper_2509_15148_b200 import binding
        sizes = (B, M, Hq, Hk, D, st["max_tokens"], st["max_len"], st["window"], st["sinks"])
        if case["op"] == "window_attention":
            st["cache"], n = binding.PagedCache(st["k"], st["v"], st["table"]), binding.window_attention_workspace_bytes(*sizes)
        else:
            st["packed"], n = binding.PackedCache(st["kp"], st["vp"], st["table"], page, D), binding.packed_attention_workspace_bytes(*sizes)
        st["workspace"] = torch.empty(n, dtype=torch.uint8, device="cuda")
    return st


# --------------------------------------------------------------------------------------------------------------------
# one pass
# --------------------------------------------------------------------------------------------------------------------
def run(st):
    if own:
        return _run_own(st)
    if st["op"] == "norm_rope_append":
        return _norm_rope_append(st)
    if st["op"] == "packed_append":
        return _packed_append(st)
    return _attend(st)


def _run_own(st):
    from paper_2509_15148_b200 import binding
    if st["op"] == "norm_rope_append":
        binding.norm_rope_append(st["q"], st["k_new"], st["v_new"], st["positions"], st["freqs"], st["q_gain"], st["k_gain"], EPS, st["cache"],
                                 st["ctx"], st["cu"], st["max_tokens"], st["q_out"], interleaved=st["interleaved"])
        return {"q": st["q_out"], "k": st["k"], "v": st["v"]}
    if st["op"] == "packed_append":
        binding.packed_append(st["k_new"], st["v_new"], st["packed"], st["ctx"], st["cu"], st["max_tokens"])
        binding.packed_read(st["packed"], st["lens"], st["max_len"], st["cache"])
        return {"k": st["k"], "v": st["v"]}
    call, cache = (binding.window_attention, st["cache"]) if st["op"] == "window_attention" else (binding.packed_attention, st["packed"])
    call(st["q"], cache, st["ctx"], st["cu"], st["pre"], st["end"], st["depth"], st["window"], st["sinks"], st["max_tokens"], st["max_len"],
         st["scale"], st["out"], st["lse"], st["workspace"])
    return {"out": st["out"], "lse": st["lse"]}


def _where(st, M):
    """(sequence, place in it) of every token."""
    cu = st["cu"].long()
    i = torch.arange(M, device="cuda")
    b = torch.searchsorted(cu, i, right=True) - 1
    return b, i - cu[b]


def _normed(x, gain):
    x = x.float()
    return x * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS) * gain.float()


def _rotate(x, c, s, half, interleaved):
    y = x.clone()
    if interleaved:
        a, b = x[..., 0 : 2 * half : 2], x[..., 1 : 2 * half : 2]
        y[..., 0 : 2 * half : 2], y[..., 1 : 2 * half : 2] = a * c - b * s, b * c + a * s
    else:
        a, b = x[..., :half], x[..., half : 2 * half]
        y[..., :half], y[..., half : 2 * half] = a * c - b * s, b * c + a * s
    return y


def _drafted(st, M):
    """(page, entry) of every drafted token's slot."""
    b, t = _where(st, M)
    slot = st["ctx"].long()[b] + t
    return st["table"].long()[b, slot // st["page"]], slot % st["page"]


def _norm_rope_append(st):
    angle = st["positions"].double()[:, None] * st["freqs"]        # far positions: 32 bits would lose the angle
    c, s = (f(angle).float()[:, None] for f in (torch.cos, torch.sin))
    half = st["freqs"].numel()
    q = _rotate(_normed(st["q"], st["q_gain"]), c, s, half, st["interleaved"]).to(st["q"].dtype)
    page, off = _drafted(st, q.shape[0])
    st["k"][page, off] = _rotate(_normed(st["k_new"], st["k_gain"]), c, s, half, st["interleaved"]).to(st["k"].dtype)
    st["v"][page, off] = st["v_new"]
    return {"q": q, "k": st["k"], "v": st["v"]}


# The cache in 4 bits.  32 neighbouring channels of a slot share a scale, a number of five exponent and three fraction bits:
# the largest magnitude over 7, at most 2048, to fp16 and then to the nearest of them (ties to even); a channel is its
# nearest whole multiple of it, -7 to 7.  A group with a value that is not finite has the scale NaN.
# A page of a head is laid out by eights of slots, 8 * D / 2 bytes of codes and 8 * D / 32 bytes of scales each.  A code c is
# held as c + 8; eight channels share a little-endian word with channel 2 i in bits 4 i and channel 2 i + 1 in bits 16 + 4 i.
_NIBBLES = (0, 4, 1, 5, 2, 6, 3, 7)


def _quantise(x):
    """(whole multiples, scales' bytes) of [..., D] in groups of 32 channels: float [..., D / 32, 32] and int [..., D / 32]."""
    x = x.float().unflatten(-1, (-1, 32))
    top = x.abs().amax(-1)
    h = torch.clamp(top / 7.0, max=2048.0).half().view(torch.int16).int()
    byte = torch.where(torch.isfinite(top), (h + 63 + ((h >> 7) & 1)) >> 7, 255)
    s = _scale(byte)[..., None]
    return torch.where(s > 0, torch.round(x / torch.where(s > 0, s, 1.0)), 0.0).clamp(-7, 7), byte


def _scale(byte):
    return (byte << 7).short().view(torch.float16).float()


def _words(code):
    """[..., D / 32, 32] whole multiples -> [..., D / 2] bytes."""
    n = (code.int() + 8).flatten(-2).unflatten(-1, (-1, 8))
    place = n[..., sorted(range(8), key=lambda c: _NIBBLES[c])]      # by nibble
    return (place[..., 0::2] | (place[..., 1::2] << 4)).to(torch.uint8).flatten(-2)


def _pack(x):
    """[pages, page, heads, D] -> [pages, heads, bytes]"""
    code, byte = _quantise(x.transpose(1, 2))
    eight = lambda t: t.unflatten(2, (-1, 8)).flatten(3)  # noqa: E731
    return torch.cat([eight(_words(code)), eight(byte.to(torch.uint8))], dim=-1).flatten(2)


def _unpack(p, page, D):
    """[pages, heads, bytes] -> float [pages, page, heads, D]"""
    p = p.unflatten(2, (page // 8, -1))
    words, byte = p[..., : 4 * D].unflatten(-1, (8, -1, 4)), p[..., 4 * D :].unflatten(-1, (8, -1))
    n = torch.stack([words & 15, words >> 4], dim=-1).flatten(-2)[..., _NIBBLES]    # [pages, heads, eights, 8, D / 8, 8]
    x = (n.float() - 8.0).flatten(-2).unflatten(-1, (-1, 32)) * _scale(byte.int())[..., None]
    return x.flatten(-2).flatten(2, 3).transpose(1, 2)


def _packed_append(st):
    M, Hk, D = st["k_new"].shape
    page, off = _drafted(st, M)
    for new, pool in ((st["k_new"], st["kp"]), (st["v_new"], st["vp"])):
        code, byte = _quantise(new)
        by_eight = pool.view(pool.shape[0], Hk, st["page"] // 8, -1)
        codes, scales = by_eight[..., : 4 * D].unflatten(-1, (8, -1)), by_eight[..., 4 * D :].unflatten(-1, (8, -1))
        codes[page, :, off // 8, off % 8] = _words(code)
        scales[page, :, off // 8, off % 8] = byte.to(torch.uint8)
    # read back: every sequence's slots
    n = st["table"].shape[1] * st["page"]
    slot = torch.arange(n, device="cuda")
    live = slot[None] < st["lens"].long()[:, None]
    page = st["table"].long()[:, slot // st["page"]][live]
    off = (slot % st["page"])[None].expand_as(live)[live]
    for pool, dst in ((st["kp"], st["k"]), (st["vp"], st["v"])):
        dst[page, off] = _unpack(pool, st["page"], D)[page, off].to(dst.dtype)
    return {"k": st["k"], "v": st["v"]}


def _attend(st):
    M, Hq, D = st["q"].shape
    B, T, S, Hk = st["ctx"].numel(), st["max_tokens"], st["max_len"], st["Hk"]
    G = Hq // Hk
    k, v = (st["k"], st["v"]) if st["op"] == "window_attention" else (_unpack(x, st["page"], D) for x in (st["kp"], st["vp"]))
    b, t = _where(st, M)
    slot = torch.arange(S, device="cuda")
    cu, ctx = st["cu"].long(), st["ctx"].long()
    n = cu[1:] - cu[:-1]
    live = slot[None] < (ctx + n)[:, None]                                   # [B, S]
    page = torch.where(live, st["table"].long()[:, slot.clamp(max=st["table"].shape[1] * st["page"] - 1) // st["page"]], 0)
    off = (slot % st["page"])[None].expand(B, S)
    q = torch.zeros(B, T, Hq, D, device="cuda")
    q[b, t] = st["q"].float()
    q = q.unflatten(2, (Hk, G)).permute(0, 2, 1, 3, 4).reshape(B, Hk, T * G, D)
    s = torch.matmul(q, k[page, off].float().permute(0, 2, 3, 1)).mul_(st["scale"])     # [B, Hk, T * G, S]
    # the tree: a drafted slot is seen by itself and its descendants; its place on their line is ctx + depth
    pre_flat, end_flat, depth = (t, n[b], t) if st["pre"] is None else (st[x].long() for x in ("pre", "end", "depth"))
    pre, mine, lo, hi = (torch.full(x, y, device="cuda") for x, y in (((B, T), -1), ((B, T), 0), ((B, S), 1 << 30), ((B, S), 0)))
    pre[b, t], mine[b, t] = pre_flat, ctx[b] + depth
    lo[b, ctx[b] + t], hi[b, ctx[b] + t] = pre_flat, end_flat
    place = slot[None].repeat(B, 1)
    place[b, ctx[b] + t] = ctx[b] + depth
    old = slot[None] < ctx[:, None]
    lo, hi = torch.where(old, 0, lo), torch.where(old, 1 << 30, hi)
    see = (lo[:, None] <= pre[:, :, None]) & (pre[:, :, None] < hi[:, None]) & live[:, None]   # [B, T, S]
    if st["window"]:
        see &= (mine[:, :, None] - place[:, None] < st["window"]) | (place < st["sinks"])[:, None]
    s.view(B, Hk, T, G, S).masked_fill_(~see[:, None, :, None], float("-inf"))
    m = s.amax(-1, keepdim=True)
    m = torch.where(m == float("-inf"), 0.0, m)
    p = s.sub_(m).exp_()
    l = p.sum(-1, keepdim=True)
    o = torch.matmul(p, torch.where(live[:, :, None, None], v[page, off].float(), 0.0).permute(0, 2, 1, 3)) / torch.where(l == 0, 1.0, l)
    rows = lambda x: x.view(B, Hk, T, G, -1)[b, :, t].flatten(1, 2)  # noqa: E731
    return {"out": rows(o).to(st["q"].dtype), "lse": rows(m + torch.log(l)).squeeze(-1).contiguous()}


# --------------------------------------------------------------------------------------------------------------------
# the work that no implementation can do without
# --------------------------------------------------------------------------------------------------------------------
def _sees(parent, ctx, window, sinks):
    """Truth values [tokens, slots]: the cache and a token's line of parents, through the window."""
    T = len(parent)
    tree, depth = np.zeros((T, T), bool), np.zeros(T, np.int64)
    for i in range(T):
        if parent[i] >= 0:
            tree[i, : parent[i] + 1], depth[i] = tree[parent[i], : parent[i] + 1], depth[parent[i]] + 1
        tree[i, i] = True
    see = np.concatenate([np.ones((T, ctx), bool), tree], axis=1)
    if window:
        place = np.concatenate([np.arange(ctx), ctx + depth])
        see &= (place[None] > (ctx + depth)[:, None] - window) | (place < sinks)[None]
    return see


def work(case):
    Hq, Hk, D = case["Hq"], case["Hk"], case["D"]
    _, tokens, ctx, parent = _batch(case, 1)
    M, row = int(tokens.sum()), D // 2 + D // 32       # a slot of one head in 4 bits
    if case["op"] == "norm_rope_append":
        return {"bytes": M * (2 * 2 * D * (Hq + 2 * Hk) + 4), "flops": M * (3 * case["rot"] + 4 * D) * (Hq + Hk)}
    if case["op"] == "packed_append":
        slots = int((tokens + ctx).sum())
        return {"bytes": 2 * Hk * (M * (2 * D + row) + slots * (row + 2 * D)), "flops": 2 * Hk * D * (5 * M + 2 * slots)}
    pairs, slots = 0, 0
    for t, c, p in zip(tokens, ctx, parent):
        if case["window"]:
            see = _sees(p, int(c), case["window"], case["sinks"])
            pairs, slots = pairs + int(see.sum()), slots + int(see.any(0).sum())
        else:
            pairs, slots = pairs + int(t) * int(c) + int((_preorder(p)[2] + 1).sum()), slots + int(t + c)
    each = 2 * D if case["op"] == "window_attention" else row
    return {"bytes": 4 * D * M * Hq + 2 * each * slots * Hk + 4 * M * Hq, "flops": 4 * D * Hq * pairs}


# --------------------------------------------------------------------------------------------------------------------
# the definitions in 64 bits
# --------------------------------------------------------------------------------------------------------------------
def exact(case, seed):
    st = prepare(case, seed)
    if case["op"] == "norm_rope_append":
        return _exact_rope(case, seed, st)
    if case["op"] == "packed_append":
        return _exact_append(case, seed, st)
    return _exact_attention(case, seed, st)


def _slots(case, seed, st):
    """For every sequence: (rows of its drafted tokens, pages and entries of their slots, of all its slots)."""
    _, tokens, ctx, _ = _batch(case, int(seed))
    table, at = st["table"].cpu().numpy().astype(np.int64), 0
    for b in range(case["B"]):
        n, c = int(tokens[b]), int(ctx[b])
        every = np.arange(c + n)
        page, off = (torch.from_numpy(x).cuda() for x in (table[b, every // case["page"]], every % case["page"]))
        yield slice(at, at + n), page[c:], off[c:], page, off
        at += n


def _exact_rope(case, seed, st):
    r = case["rot"]
    angle = st["positions"].double()[:, None] * st["freqs"]
    turn = torch.polar(torch.ones_like(angle), angle)[:, None]      # one complex number per pair

    def turned(x, gain):
        x = x.double()
        x = x / torch.sqrt(x.square().sum(-1, keepdim=True) / x.shape[-1] + EPS) * gain.double()
        z = x[..., :r].unflatten(-1, (r // 2, 2)) if case["layout"] == "interleaved" else x[..., :r].unflatten(-1, (2, r // 2)).transpose(-1, -2)
        z = torch.view_as_real(torch.view_as_complex(z.contiguous()) * turn)
        z = z if case["layout"] == "interleaved" else z.transpose(-1, -2)
        return torch.cat([z.flatten(-2), x[..., r:]], dim=-1)

    q, k = turned(st["q"], st["q_gain"]), turned(st["k_new"], st["k_gain"])
    kc, vc = st["k"].double(), st["v"].double()
    for rows, page, off, _, _ in _slots(case, seed, st):
        kc[page, off], vc[page, off] = k[rows], st["v_new"][rows].double()
    return {"q": q, "k": kc, "v": vc}


def _numbers():
    """The 255 scales that are numbers, in order: eight fractions for each exponent."""
    return torch.tensor([m * 2.0 ** -17 for m in range(8)] + [(8 + m) * 2.0 ** (e - 18) for e in range(1, 32) for m in range(8)][:247], dtype=torch.float64)


def _in_four_bits(x):
    """x [..., D] as the cache holds it."""
    x = x.double().unflatten(-1, (-1, 32))
    a = (x.abs().amax(-1) / 7.0).clamp(max=2048.0).half().double()
    scales = _numbers().cuda()
    up = torch.searchsorted(scales, a).clamp(1, 254)
    low, high = scales[up - 1], scales[up]
    s = torch.where((a - low < high - a) | ((a - low == high - a) & ((up - 1) % 2 == 0)), low, high)[..., None]
    near = torch.round(x / torch.where(s > 0, s, 1.0))
    return torch.where(s > 0, near.clamp(-7, 7) * s, 0.0).flatten(-2)


def _values(pool, page, D):
    """What a packed pool [pages, heads, bytes] stands for, by its layout: fp64 [pages, heads, page, D]."""
    eights = pool.reshape(pool.shape[0], pool.shape[1], page // 8, -1)
    word = eights[..., : 4 * D].contiguous().view(torch.int32).reshape(*eights.shape[:3], 8, D // 8)
    at = torch.tensor([4 * (c // 2) + 16 * (c % 2) for c in range(8)], device=pool.device, dtype=torch.int32)
    code = ((word[..., None] >> at) & 15).double() - 8.0
    scale = torch.cat([_numbers().to(pool.device), torch.full((1,), float("nan"), dtype=torch.float64, device=pool.device)])[eights[..., 4 * D :].long()]
    scale = scale.reshape(*eights.shape[:3], 8, D // 32)
    return (code.reshape(*scale.shape, 32) * scale[..., None]).flatten(-2).flatten(2, 3)


def _exact_append(case, seed, st):
    out = []
    for new, pool, dst in ((st["k_new"], st["kp"], st["k"]), (st["v_new"], st["vp"], st["v"])):
        held, got = _values(pool, case["page"], case["D"]).transpose(1, 2), dst.double()
        for rows, page, off, every_page, every_off in _slots(case, seed, st):
            got[every_page, every_off] = held[every_page, every_off]
            got[page, off] = _in_four_bits(new[rows])
        out.append(got)
    return {"k": out[0], "v": out[1]}


def _exact_attention(case, seed, st):
    _, tokens, ctx, parent = _batch(case, int(seed))
    Hq, Hk, D, page = case["Hq"], case["Hk"], case["D"], case["page"]
    G, M = Hq // Hk, st["q"].shape[0]
    out, lse = torch.zeros(M, Hq, D, dtype=torch.float64, device="cuda"), torch.zeros(M, Hq, dtype=torch.float64, device="cuda")
    at = 0
    for b in range(case["B"]):
        n, S = int(tokens[b]), int(tokens[b] + ctx[b])
        see = torch.from_numpy(_sees(parent[b], int(ctx[b]), case["window"], case["sinks"])).cuda()
        pages = st["table"][b, : -(-S // page)].long()
        for h in range(Hk):
            if case["op"] == "window_attention":
                k, v = (st[x][pages, :, h].flatten(0, 1)[:S].double() for x in ("k", "v"))
            else:
                k, v = (_values(st[x][pages, h : h + 1], page, D)[:, 0].flatten(0, 1)[:S] for x in ("kp", "vp"))
            for g in range(h * G, (h + 1) * G):
                s = (st["q"][at : at + n, g].double() @ k.T) * st["scale"]
                s[~see] = float("-inf")
                lse[at : at + n, g] = torch.logsumexp(s, -1)
                out[at : at + n, g] = torch.softmax(s, -1) @ v
        at += n
    return {"out": out, "lse": lse}
