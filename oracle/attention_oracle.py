"""Plain fp64 numpy statement of the attention side: rotary positions and append, attention of drafted trees over a paged
cache, attention weight per cached slot, selection and move of an eviction.  One sequence, token and head at a time, from
the definitions; shares no code with the CUDA library.

Caches are numpy arrays [num_pages, page_size, heads, head_dim]; `table` [num_seqs, pages]; slot s of sequence b is entry
s % page_size of page table[b, s // page_size]; drafted token t of sequence b has slot ctx[b] + t."""
from __future__ import annotations

import math

import numpy as np


def rotate(x, position: int, freqs, mscale: float = 1.0, interleaved: bool = False):
    """x [..., head_dim] float64 with its first 2 * len(freqs) channels turned pair by pair by position * freqs."""
    x = np.asarray(x, np.float64)
    out = x.copy()
    half = len(freqs)
    for i, f in enumerate(freqs):
        a = math.fmod(float(position) * float(f), 2 * math.pi)
        c, s = mscale * math.cos(a), mscale * math.sin(a)
        p, r = (2 * i, 2 * i + 1) if interleaved else (i, half + i)
        out[..., p] = x[..., p] * c - x[..., r] * s
        out[..., r] = x[..., r] * c + x[..., p] * s
    return out


def visible(parent, t: int) -> list[int]:
    """Drafted tokens that token t of a tree sees: itself and its line of parents; nothing if it is padding (-2)."""
    line = []
    if parent[t] == -2:
        return line
    while t >= 0:
        line.append(t)
        t = int(parent[t])
    return line[::-1]


def cached(cache, table_row, slots, head: int):
    """Rows of a paged cache [len(slots), head_dim] in float64."""
    page_size = cache.shape[1]
    return np.array([cache[table_row[s // page_size], s % page_size, head] for s in slots], np.float64).reshape(len(slots), cache.shape[3])


def tree_attention(q, k, v, table, ctx, cu, parent, scale: float):
    """q [M, Hq, D]; parent [M] within each sequence -> out [M, Hq, D], lse [M, Hq] (0 and -inf where nothing is seen)."""
    M, Hq, D = q.shape
    G = Hq // k.shape[2]
    out, lse = np.zeros((M, Hq, D)), np.full((M, Hq), -np.inf)
    for b in range(len(ctx)):
        par = parent[cu[b]:cu[b + 1]]
        for t in range(len(par)):
            drafts = visible(par, t)
            if not drafts:
                continue
            slots = list(range(ctx[b])) + [ctx[b] + j for j in drafts]
            for h in range(k.shape[2]):
                kk, vv = cached(k, table[b], slots, h), cached(v, table[b], slots, h)
                s = np.asarray(q[cu[b] + t, h * G:(h + 1) * G], np.float64) @ kk.T * scale
                m = s.max(-1, keepdims=True)
                p = np.exp(s - m)
                l = p.sum(-1, keepdims=True)
                out[cu[b] + t, h * G:(h + 1) * G] = p @ vv / l
                lse[cu[b] + t, h * G:(h + 1) * G] = (m + np.log(l))[:, 0]
    return out, lse


def cache_weights(q, k, table, lse, ctx, cu, parent, scale: float, cols: int):
    """[num_seqs, heads, cols]: what every slot receives, given each row's lse."""
    Hq = q.shape[1]
    G = Hq // k.shape[2]
    w = np.zeros((len(ctx), k.shape[2], cols))
    for b in range(len(ctx)):
        par = parent[cu[b]:cu[b + 1]]
        for t in range(len(par)):
            drafts = visible(par, t)
            if not drafts:
                continue
            slots = list(range(ctx[b])) + [ctx[b] + j for j in drafts]
            for h in range(k.shape[2]):
                s = np.asarray(q[cu[b] + t, h * G:(h + 1) * G], np.float64) @ cached(k, table[b], slots, h).T * scale
                w[b, h, slots] += np.exp(s - np.asarray(lse[cu[b] + t, h * G:(h + 1) * G], np.float64)[:, None]).sum(0)
    return w


def select(weights, length: int, budget: int, sinks: int, recent: int) -> list[int]:
    """Slots of one row that an eviction keeps, ascending; a NaN weight is below every number."""
    if length <= budget:
        return list(range(length))
    def order(i):
        forced = i < sinks or i >= length - recent
        w = float(weights[i])
        return (not forced, math.isnan(w), 0.0 if math.isnan(w) else -w, i)
    return sorted(sorted(range(length), key=order)[:budget])
