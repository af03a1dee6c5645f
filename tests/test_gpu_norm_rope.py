"""Normed rotations on the device against the fp64 definition.

Tolerance.  A normed channel: the sum of at most 256 squares by threads (16 each) and a tree is off by 20 * 2^-24 of itself, its root by
half of that, the approximate reciprocal root by 2 * 2^-24, three products by half a step each: 14 * 2^-24 < 1e-6 of it.
Cosine and sine: 2 units in the last place and an argument of half a turn at most rounded to 24 bits: 4e-7.  A turned channel of a pair
(a, b) is so off by 2e-6 (|a| + |b|) |mscale| <= d = 4e-6 max |row| |mscale|, and the rounding to the output adds u (|y| + d)."""
import numpy as np
import pytest
import torch

from oracle import window_packed_oracle as orc
from paper_2509_15148_b200 import binding

pytestmark = pytest.mark.gpu
BF, FP = torch.bfloat16, torch.float16
UNIT = {BF: 2.0 ** -8, FP: 2.0 ** -11}
EPS = 1e-5


def i32(x):
    return torch.as_tensor(np.asarray(x), dtype=torch.int32).cuda()


def rows(g, M, heads, D, dtype, pad, scale=3.0):
    """[M, heads, D] as a view whose rows are `pad` elements longer."""
    t = (torch.randn(M, heads, D + pad, generator=g, device="cuda") * scale).to(dtype)
    return t[..., :D]


def check(got, x, gain, pos, freqs, mscale, inter, dtype):
    x, got = x.double().cpu().numpy(), got.double().cpu().numpy()
    gain = None if gain is None else gain.double().cpu().numpy()
    for t in range(x.shape[0]):
        want = orc.norm_rotate(x[t], gain, EPS, int(pos[t]), freqs, mscale, inter)
        before = orc.norm_rotate(x[t], gain, EPS, 0, [], 1.0)
        d = 4e-6 * np.abs(before).max(-1, keepdims=True) * max(1.0, abs(mscale))
        assert (np.abs(got[t] - want) <= d + UNIT[dtype] * (np.abs(want) + d)).all(), np.abs(got[t] - want).max()


CASES = [  # D, pairs, interleaved, dtype, Hq, Hk, row padding, gains, tokens
    (64, 32, False, BF, 4, 2, 0, True, [3, 0, 2]),
    (128, 64, False, FP, 8, 1, 0, True, [1]),
    (128, 32, True, BF, 5, 5, 8, True, [7, 1]),
    (256, 128, False, BF, 2, 1, 0, True, [4]),
    (256, 64, True, FP, 3, 3, 16, True, [4]),
    (96, 16, False, FP, 2, 2, 0, True, [5]),
    (24, 8, False, BF, 2, 1, 0, True, [5]),          # three pieces of a row
    (8, 4, True, BF, 1, 1, 0, True, [5]),
    (80, 0, False, BF, 2, 1, 0, True, [5]),          # norm alone
    (128, 64, False, BF, 4, 2, 1, True, [6, 3]),     # rows that are not aligned
    (72, 13, False, FP, 3, 1, 3, True, [6]),         # pairs that do not fill pieces
    (72, 13, True, BF, 3, 1, 0, True, [6]),
    (128, 64, False, BF, 4, 2, 0, False, [9]),       # neither side normed
    (128, 64, False, FP, 4, 2, 0, "k", [9]),         # keys alone
    (128, 64, False, BF, 40, 8, 0, True, [500, 1, 733]),
]


@pytest.mark.parametrize("case", CASES)
def test_append_and_rows_against_the_definition(case):
    D, pairs, inter, dtype, Hq, Hk, pad, gains, tokens = case
    g = torch.Generator(device="cuda").manual_seed(7)
    rs = np.random.RandomState(7)
    M, B, page = sum(tokens), len(tokens), 16
    big = M > 100
    q, k, v = rows(g, M, Hq, D, dtype, pad), rows(g, M, Hk, D, dtype, pad), rows(g, M, Hk, D, dtype, pad)
    qg = (1 + 0.5 * torch.randn(D, generator=g, device="cuda")).to(dtype) if gains is True else None
    kg = (1 + 0.5 * torch.randn(D, generator=g, device="cuda")).to(dtype) if gains else None
    freqs = torch.from_numpy(rs.rand(pairs) ** 3)
    pos = rs.randint(0, 1 << 20, M)
    mscale = 1.25
    ctx = rs.randint(0, 40, B)
    need = -(-(ctx + np.array(tokens)) // page)
    table = rs.permutation(int(need.sum())).astype(np.int64)
    tab = np.full((B, int(need.max())), -1)
    at = 0
    for b in range(B):
        tab[b, :need[b]] = table[at:at + need[b]]
        at += need[b]
    kc, vc = (torch.full((int(need.sum()), page, Hk, D), 9.0, dtype=dtype, device="cuda") for _ in range(2))
    cache = binding.PagedCache(kc, vc, i32(tab))
    cu = np.concatenate([[0], np.cumsum(tokens)])
    out = torch.empty(M, Hq, D, dtype=dtype, device="cuda")
    turn = (i32(pos), freqs.cuda(), qg, kg, EPS)
    binding.norm_rope_append(q, k, v, *turn, cache, i32(ctx), i32(cu), max(tokens), out, interleaved=inter, mscale=mscale)
    at = rs.choice(M, 40, replace=False) if big else np.arange(M)
    seq = np.searchsorted(cu, at, side="right") - 1
    slot = ctx[seq] + at - cu[seq]
    pages, offs = torch.as_tensor(tab[seq, slot // page]).cuda(), torch.as_tensor(slot % page).cuda()
    idx = torch.as_tensor(at).cuda()
    check(out[idx], q[idx], qg, pos[at], freqs.numpy(), mscale, inter, dtype)
    check(kc[pages, offs], k[idx], kg, pos[at], freqs.numpy(), mscale, inter, dtype)
    assert torch.equal(vc[pages, offs], v[idx])
    assert int((kc == 9.0).all(-1).all(-1).sum()) == kc.shape[0] * page - M      # every other slot as it was
    # rows to rows, the keys in place: the same bits
    out2, kin = torch.empty_like(out), k.clone()
    binding.norm_rope(q, kin, *turn, out2, kin, interleaved=inter, mscale=mscale)
    assert torch.equal(out2, out) and torch.equal(kin[idx], kc[pages, offs])
    if pad == 0 or D % 8 == 0 and pad % 8 == 0:
        qin = q.clone(memory_format=torch.preserve_format)
        binding.norm_rope(qin, None, *turn, qin, None, interleaved=inter, mscale=mscale)
        assert torch.equal(qin, out)
    assert binding.last_device_status() == 0


def test_zeros_special_values_and_bad_sequences():
    D, page = 64, 8
    x = torch.zeros(3, 1, D, dtype=BF, device="cuda")
    x[1] = float("nan")
    x[2, 0, 5] = 1e15
    freqs, pos, gain = torch.full((32,), 0.1, dtype=torch.float64).cuda(), i32([5, 6, 7]), torch.ones(D, dtype=BF, device="cuda")
    kc, vc = (torch.full((2, page, 1, D), 3.0, dtype=BF, device="cuda") for _ in range(2))
    cache = binding.PagedCache(kc, vc, i32([[0], [7]]))
    out = torch.empty_like(x)
    binding.norm_rope_append(x, x, x, pos, freqs, gain, gain, EPS, cache, i32([0, 0]), i32([0, 2, 3]), 2, out)
    assert (out[0] == 0).all() and torch.isnan(out[1]).all()
    turned = orc.norm_rotate(x[2].double().cpu().numpy(), np.ones(D), EPS, 7, [0.1] * 32)
    assert np.abs(out[2].double().cpu().numpy() - turned).max() <= 2.0 ** -8 * 8.01
    assert (kc[0, 0] == 0).all() and torch.isnan(kc[0, 1]).all() and (kc[0, 2:] == 3).all() and (kc[1] == 3).all()   # page 7 is none: not written
    assert binding.last_device_status() == binding.DEV_PAGE_RANGE
    out.fill_(5)
    binding.norm_rope_append(x, x, x, pos, freqs, gain, gain, EPS, cache, i32([-1, 0]), i32([0, 2, 3]), 1, out)
    assert (out[:2] == 5).all() and binding.last_device_status() & binding.DEV_SEQ_RANGE     # a negative length: left out
    binding.norm_rope(x[:0], x[:0], pos[:0], freqs, gain, gain, EPS, x[:0], x[:0])
    assert binding.last_device_status() == 0
