"""Plain fp64 numpy statement of the normed rotation, of attention through a window, and of the cache in 4 bits; one row, token or
group at a time, from the definitions.  Shares no code with the CUDA library."""
from __future__ import annotations

import math

import numpy as np

from oracle.attention_oracle import rotate, visible


def norm_rotate(x, gain, eps: float, position: int, freqs, mscale: float = 1.0, interleaved: bool = False):
    """x [..., head_dim] / sqrt(mean(x^2) + eps) * gain, then turned; gain None: only turned."""
    x = np.asarray(x, np.float64)
    if gain is not None:
        x = x / np.sqrt((x * x).mean(-1, keepdims=True) + eps) * np.asarray(gain, np.float64)
    return rotate(x, position, freqs, mscale, interleaved)


def sees(parent, ctx: int, window: int = 0, sinks: int = 0):
    """Truth values [tokens, ctx + tokens]: what each drafted token of one sequence sees; window 0: everything on its line."""
    T = len(parent)
    out = np.zeros((T, ctx + T), bool)
    lines = [visible(parent, t) for t in range(T)]
    for t, line in enumerate(lines):
        if not line:
            continue
        items = [(s, s) for s in range(ctx)] + [(ctx + j, ctx + len(lines[j]) - 1) for j in line]     # (slot, place)
        mine = ctx + len(line) - 1
        for slot, place in items:
            out[t, slot] = window == 0 or mine - place < window or place < sinks
    return out


# ---- the cache in 4 bits ----------------------------------------------------------------------------------------------
def scale_of(byte: int) -> float:
    """The number of five exponent and three fraction bits that a byte stands for; 208 (2048) is the largest that is one."""
    if byte > 208:
        return math.nan
    e, f = byte >> 3, byte & 7
    return f * 2.0 ** -17 if e == 0 else (8 + f) * 2.0 ** (e - 18)


_SCALES = np.array([scale_of(b) for b in range(209)])


def quantise(group):
    """(byte, 32 whole multiples) of a group of 32 channels."""
    g = np.asarray(group, np.float64)
    if not np.isfinite(g).all():
        return 255, np.zeros(32, np.int64)
    top = float(np.float16(min(np.abs(g).max() / 7, 2048.0)))       # (rounded twice, as the format has it)
    byte = int(np.searchsorted(_SCALES, top))
    if _SCALES[byte] > top:                # between byte - 1 and byte: the nearer, at a tie the even one
        low, high = top - _SCALES[byte - 1], _SCALES[byte] - top
        if low < high or (low == high and byte % 2 == 1):
            byte -= 1
    s = _SCALES[byte]
    if s == 0:
        return byte, np.zeros(32, np.int64)
    return byte, np.clip([round(x / s) for x in g.tolist()], -7, 7).astype(np.int64)      # (Python rounds ties to even)


def packed_slot(x):
    """(codes, scales) of one slot [head_dim] as bytes."""
    codes, scales = [], []
    for g in range(0, len(x), 32):
        byte, c = quantise(x[g:g + 32])
        scales.append(byte)
        for w in range(0, 32, 8):
            word = 0
            for j in range(8):
                word |= int(c[w + j] + 8) << (4 * (j // 2) + 16 * (j % 2))
            codes += [(word >> (8 * b)) & 255 for b in range(4)]
    return np.array(codes, np.uint8), np.array(scales, np.uint8)


def slot_bytes(entry: int, D: int):
    """(first byte of the codes, of the scales) of an entry within its page's block of a head."""
    piece = entry // 8 * (4 * D + D // 4)
    return piece + entry % 8 * (D // 2), piece + 4 * D + entry % 8 * (D // 32)


def unpack(block, page_size: int, D: int):
    """Values [page_size, D] of a block of bytes."""
    out = np.zeros((page_size, D))
    for e in range(page_size):
        c0, s0 = slot_bytes(e, D)
        for w in range(D // 8):
            word = sum(int(block[c0 + 4 * w + b]) << (8 * b) for b in range(4))
            s = scale_of(int(block[s0 + w // 4]))
            for j in range(8):
                out[e, 8 * w + j] = (((word >> (4 * (j // 2) + 16 * (j % 2))) & 15) - 8) * s
    return out
