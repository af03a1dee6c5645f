"""Windowed and packed attention at their edges, in every form that a call may take: sequences of padding alone, pages that are gone or
missing, infinities and NaN, the smallest scales and scores beyond fp32, thousands of sequences; the packed cache's small groups and
the ends of the norm's range.

A call's form goes by the rows that a sequence's key head can have (drafted tokens times the query heads that share it): over a packed
cache up to 8 and up to 16, in both up to 64, up to 128, more; over 16 bits also many short sequences.  ROWS has a batch of each.
Tolerances are those of test_gpu_attention.py."""
import numpy as np
import pytest
import torch

from oracle import window_packed_oracle as orc
from paper_2509_15148_b200 import binding
from tests.test_gpu_attention import BF, FP, i32
from tests.test_gpu_window_packed import Windowed, pack_pool

pytestmark = pytest.mark.gpu

ROWS = {  # tokens of the longest sequence, Hq, Hk
    "8": (4, 4, 2), "16": (4, 8, 2), "64": (20, 4, 2), "128": (100, 2, 2), "more": (200, 4, 2),
}


def made(packed, change, *args, **kw):
    """A batch whose cache `change` has altered before it is packed."""
    b = Windowed(*args, **kw)
    change(b)
    if packed:
        b.packed, b.pools = True, []
        for name in ("k", "v"):
            pool, value = pack_pool(getattr(b, name))
            b.pools.append(pool)
            setattr(b, name, value)
        b.handle = binding.PackedCache(*b.pools, b.table, b.page, b.D)
    return b


def others(b, out, lse, want, hit):
    """Rows outside `hit` (truth values [M, Hq]) are right; those in it are NaN."""
    assert torch.isnan(lse[hit]).all() and torch.isnan(out[hit]).all()
    fine = ~hit
    out, lse = out.clone(), lse.clone()
    out[hit], lse[hit] = want[0][hit].to(out.dtype), want[1][hit].float()
    assert fine.any()
    b.check(out, lse, *want)


# ---- sequences of padding alone -----------------------------------------------------------------------------------------
@pytest.mark.parametrize("packed, window, sinks", [(False, 50, 4), (True, 0, 0), (True, 50, 4), (True, 3000, 0)])
@pytest.mark.parametrize("rows", ROWS)
@pytest.mark.parametrize("ctx", [[70, 300, 40], [5000, 6000, 300]])
def test_a_sequence_of_padding_alone_needs_no_page(rows, ctx, packed, window, sinks):
    n, Hq, Hk = ROWS[rows]
    b = Windowed(11, [n, n, 1], ctx, Hq, Hk, 128, 16, BF, "random", 0.0, window=window, sinks=sinks, packed=packed)
    b.parent[n:2 * n] = -2
    pre, end, depth = binding.tree_plan(b.parent, b.cu_h)
    b.pre, b.end, b.depth = pre.cuda(), end.cuda(), depth.cuda()
    want = b.dense()
    b.table[1] = -1
    assert binding.last_device_status() == 0
    out, lse = b.call()
    assert binding.last_device_status() == 0
    b.check(out, lse, *want)
    assert (out[n:2 * n] == 0).all() and (lse[n:2 * n] == -float("inf")).all()


# ---- pages ----------------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("packed", [False, True])
@pytest.mark.parametrize("page", [8, 16, 256])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("rows", list(ROWS) + ["many"])
def test_pages_behind_the_window_may_be_gone_in_every_form(rows, D, page, packed):
    n, Hq, Hk = ROWS.get(rows, (1, 8, 2))
    tokens, ctx = ([1] * 148, [640 + i for i in range(148)]) if rows == "many" else ([n, 1, 2], [1000, 1640, 777])
    b = Windowed(12, tokens, ctx, Hq, Hk, D, page, FP, "random", 0.0, window=100, sinks=5, packed=packed)
    want = b.dense()
    for i in range(b.B):
        cols = np.arange(b.table.shape[1])
        gone = (page * cols >= 5) & (page * cols + page <= int(b.ctx_h[i]) - 100 + 1)
        assert gone.any()
        b.table[i, torch.from_numpy(gone).cuda()] = -1
    assert binding.last_device_status() == 0
    out, lse = b.call()
    assert binding.last_device_status() == 0
    b.check(out, lse, *want)


@pytest.mark.parametrize("window", [0, 300])
@pytest.mark.parametrize("page", [8, 64])
@pytest.mark.parametrize("rows", ROWS)
def test_packed_pages_that_are_missing_read_as_zeros_in_every_form(rows, page, window):
    n, Hq, Hk = ROWS[rows]
    b = Windowed(13, [n, 2], [400, 150], Hq, Hk, 64, page, BF, "random", 0.0, window=window, sinks=2 if window else 0, packed=True)
    for col in (200 // page, 390 // page):
        for x in (b.k, b.v):
            x[b.table[0, col].item()] = 0
    want = b.dense()
    b.table[0, 200 // page], b.table[0, 390 // page] = b.n_pages, -7
    assert binding.last_device_status() == 0
    out, lse = b.call()
    assert binding.last_device_status() == binding.DEV_PAGE_RANGE
    b.check(out, lse, *want)


# ---- infinities and NaN -----------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("packed, window", [(False, 200), (False, 9000), (True, 0), (True, 200), (True, 9000)])
@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("ctx", [300, 20000])
@pytest.mark.parametrize("rows", ROWS)
def test_infinite_scores_reach_their_row_alone(rows, ctx, dtype, packed, window):
    """A query of zeros and one +inf, keys of 3 or -3 in that channel: scores of +inf and -inf and nothing else."""
    n, Hq, Hk = ROWS[rows]

    def change(b):
        live = ~torch.isnan(b.k[..., 0])
        sign = torch.randn(b.k[..., 0].shape, generator=torch.Generator(device="cuda").manual_seed(1), device="cuda").sign()
        b.k[..., 0] = torch.where(live, 3 * sign, b.k[..., 0].float()).to(b.dtype)
    b = made(packed, change, 14, [n, 1], [ctx, 130], Hq, Hk, 64, 32, dtype, "chain", 0.0, window=window, sinks=1)
    want = b.dense()
    b.q[1, 1] = 0
    b.q[1, 1, 0] = float("inf")
    out, lse = b.call()
    assert binding.last_device_status() == 0
    hit = torch.zeros(b.M, b.Hq, dtype=torch.bool, device="cuda")
    hit[1, 1] = True
    others(b, out, lse, want, hit)


@pytest.mark.parametrize("packed", [False, True])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("where", ["edge", "sink", "draft"])
@pytest.mark.parametrize("rows", ROWS)
def test_nan_in_a_key_reaches_the_rows_whose_window_holds_it(rows, where, D, packed):
    n, Hq, Hk = ROWS[rows]
    ctx, window, sinks = 700, 150, 3
    slot = {"edge": ctx - window + 3, "sink": 1, "draft": ctx + 1}[where]     # (the edge: seen by tokens 0, 1 and 2)

    def change(b):
        b.k[b.table_h[0, slot // b.page], slot % b.page, 1, D - 1] = float("nan")
    b = made(packed, change, 15, [n, 3], [ctx, 200], Hq, Hk, D, 16, BF, "chain", 0.0, window=window, sinks=sinks)
    want = b.dense() if packed else None
    if not packed:
        k = b.k.clone()
        b.k.nan_to_num_(0.0)
        want = b.dense()
        b.k.copy_(k)
    out, lse = b.call()
    assert binding.last_device_status() == 0
    hit = torch.zeros(b.M, b.Hq, dtype=torch.bool, device="cuda")
    hit[:n, Hq // Hk:] = torch.from_numpy(b.see(0)[:, slot]).cuda()[:, None]
    assert hit.any()
    others(b, out, lse, want, hit)


@pytest.mark.parametrize("window", [0, 150])
@pytest.mark.parametrize("what", [float("nan"), float("inf")])
@pytest.mark.parametrize("rows", ROWS)
def test_a_packed_value_that_is_not_finite_reaches_its_channels_of_rows_that_see_it(rows, what, window):
    """A group of 32 channels becomes NaN: in out of the rows that see it (what other rows of that head get is left open), not in lse, in
    other channels, heads or sequences."""
    n, Hq, Hk = ROWS[rows]
    ctx = 700

    def change(b):
        b.v[b.table_h[0, 699 // 16], 699 % 16, 0, 40] = what
    b = made(True, change, 16, [n, 3], [ctx, 200], Hq, Hk, 128, 16, FP, "chain", 0.0, window=window, sinks=0)
    want = b.dense()
    out, lse = b.call()
    assert binding.last_device_status() == 0
    sees = torch.from_numpy(b.see(0)[:, 699]).cuda()
    G = Hq // Hk
    assert torch.isnan(out[:n][sees][:, :G, 32:64]).all()
    out = out.clone()
    out[:n, :G, 32:64] = want[0][:n, :G, 32:64].to(FP)
    b.check(out, lse, *want)


# ---- the smallest scales ----------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("packed", [False, True])
@pytest.mark.parametrize("scale", [1e-38, 1e-40])
@pytest.mark.parametrize("tokens, Hq, Hk", [(4, 4, 4), (4, 16, 4), (20, 8, 4), (100, 4, 4), (200, 4, 4)])
def test_smallest_scales_weigh_all_that_is_seen_alike(tokens, Hq, Hk, scale, packed):
    """The window's edge lies so that the first 32 slots of which token 0 sees one show the others none."""
    B = 75 if tokens == 4 else 2
    b = Windowed(17, [tokens] * B, [1000] * B, Hq, Hk, 64, 16, BF, "chain", 0.0, window=1000 + 1 - 159, sinks=0, packed=packed)
    b.scale = scale
    out, lse = b.call()
    assert binding.last_device_status() == 0
    b.check(out, lse, *b.dense())


# ---- scores beyond fp32 -------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("ctx", [300, 20000])
@pytest.mark.parametrize("form", ["tree", "window", "packed", "packed window"])
@pytest.mark.parametrize("rows", ROWS)
def test_scores_that_the_scale_takes_beyond_fp32_are_not_an_empty_row(rows, form, ctx):
    """One query's products are 1.5e18 to 3e18 in size, of either sign, times a scale of 1e21: +inf in fp32, so out and lse are NaN as for
    any +inf.  The other queries are zeros: every slot that they see weighs alike."""
    n, Hq, Hk = ROWS[rows]

    def change(b):
        live = ~torch.isnan(b.k[..., 0])
        sign = torch.randn(b.k[..., 0].shape, generator=torch.Generator(device="cuda").manual_seed(1), device="cuda").sign()
        b.k[..., 0] = torch.where(live, 3 * sign, b.k[..., 0].float()).to(b.dtype)
    b = made("packed" in form, change, 19, [n, 1], [ctx, 130], Hq, Hk, 64, 32, BF, "chain", 0.0, window=200 if "window" in form else 0, sinks=1)
    b.q.zero_()
    b.scale = 1e21
    want = b.dense()[:2]
    b.q[1, 1, 0] = 1e18
    out, lse = b.attend() if form == "tree" else b.call()
    assert binding.last_device_status() == 0
    hit = torch.zeros(b.M, b.Hq, dtype=torch.bool, device="cuda")
    hit[1, 1] = True
    others(b, out, lse, want, hit)


# ---- thousands of sequences ---------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("B", [600, 1300, 5000, 9600])
@pytest.mark.parametrize("D", [64, 256])
def test_normed_rotation_of_many_sequences_of_one_token(B, D):
    """The append gives the bits that rows to rows gives, whatever the sequences."""
    g = torch.Generator(device="cuda").manual_seed(B)
    rs = np.random.RandomState(B)
    q, k, v = (torch.randn(B, h, D, generator=g, device="cuda").to(BF) for h in (4, 2, 2))
    gain = (1 + 0.3 * torch.randn(2, D, generator=g, device="cuda")).to(BF)
    freqs = binding.rope_freqs(D, 10000.0)[0].cuda()
    ctx = rs.randint(0, 8, B)
    page = rs.permutation(B)
    kc, vc = (torch.full((B, 8, 2, D), 9.0, dtype=BF, device="cuda") for _ in range(2))
    q1, q2, k2 = torch.empty_like(q), torch.empty_like(q), torch.empty_like(k)
    turn = (i32(rs.randint(0, 5000, B)), freqs, gain[0], gain[1], 1e-6)
    binding.norm_rope_append(q, k, v, *turn, binding.PagedCache(kc, vc, i32(page[:, None])), i32(ctx), i32(np.arange(B + 1)), 1, q1)
    binding.norm_rope(q, k, *turn, q2, k2)
    at = torch.from_numpy(page).cuda(), torch.from_numpy(ctx).cuda()
    assert torch.equal(q1, q2) and torch.equal(kc[at], k2) and torch.equal(vc[at], v)
    assert int((kc == 9).all(-1).all(-1).sum()) == 7 * B and binding.last_device_status() == 0
    x = orc.norm_rotate(k[B - 1].double().cpu().numpy(), gain[1].double().cpu().numpy(), 1e-6, int(turn[0][B - 1]), freqs.cpu().numpy())
    assert (np.abs(k2[B - 1].double().cpu().numpy() - x) <= 2.0 ** -8 * np.abs(x) + 4e-6 * np.abs(x).max() * 2).all()


@pytest.mark.parametrize("B", [700, 3000])
def test_packed_append_and_attention_of_many_sequences_of_one_token(B):
    rs = np.random.RandomState(B)
    b = Windowed(18, [1] * B, rs.randint(0, 40, B).tolist(), 4, 2, 64, 8, FP, "chain", 0.0, packed=True)
    new = torch.randn(2, B, 2, 64, generator=torch.Generator(device="cuda").manual_seed(2), device="cuda").half()
    at = torch.from_numpy(b.table_h[np.arange(B), b.ctx_h // 8]).cuda(), torch.from_numpy(b.ctx_h % 8).cuda()
    binding.packed_append(new[0], new[1], b.handle, b.ctx, b.cu, 1)
    for i, x in enumerate((b.k, b.v)):
        x[at] = pack_pool(new[i][:, None].repeat(1, 8, 1, 1))[1][:, 0]
    out, lse = b.call()
    assert binding.last_device_status() == 0
    b.check(out, lse, *b.dense())


# ---- the format ---------------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", [BF, FP])
def test_append_of_small_groups_is_the_format_to_the_byte(dtype):
    """Scales below 2^-14 have fewer digits: every largest magnitude up to 7 * 2^-13 in one group or another."""
    top = torch.arange(1 << 15, dtype=torch.int32).to(torch.int16).view(dtype)
    top = top[(top > 0) & (top < 7 * 2.0 ** -13)]
    top = top[-(16 * 2048):]
    n = -(-top.numel() // 16) * 16
    g = torch.Generator().manual_seed(3)
    x = (2 * torch.rand(n, 32, generator=g) - 1)
    x[: top.numel()] *= top.float()[:, None]
    x = x.to(dtype)
    x[torch.arange(top.numel()), torch.randint(0, 32, (top.numel(),), generator=g)] = top
    x = x.view(n // 2, 1, 64).cuda()
    page, slots = 256, n // 2
    pages = -(-slots // page)
    pools = [torch.full((pages, 1, binding.packed_block_bytes(page, 64)), 0xAA, dtype=torch.uint8, device="cuda") for _ in range(2)]
    binding.packed_append(x, -x, binding.PackedCache(*pools, i32(np.arange(pages)[None]), page, 64), i32([0]), i32([0, slots]), slots)
    for new, pool in ((x, pools[0]), (-x, pools[1])):
        full = torch.zeros(pages * page, 1, 64, dtype=dtype, device="cuda")
        full[:slots] = new
        want = pack_pool(full.view(pages, page, 1, 64))[0]
        whole = slots // page
        assert torch.equal(pool[:whole], want[:whole])
        for s in range(whole * page, slots):
            c0, s0 = orc.slot_bytes(s % page, 64)
            assert torch.equal(pool[whole, 0, c0:c0 + 32], want[whole, 0, c0:c0 + 32]) and torch.equal(pool[whole, 0, s0:s0 + 2], want[whole, 0, s0:s0 + 2])
    assert binding.last_device_status() == 0


# ---- the norm's range ---------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("size", [1e-17, 1e18])
@pytest.mark.parametrize("D, pad", [(64, 0), (256, 0), (256, 3)])
def test_norm_without_eps_at_the_ends_of_its_range(D, pad, size):
    """Rows of one channel of that size and of all channels near it; the tolerance of test_gpu_norm_rope.py."""
    g = torch.Generator(device="cuda").manual_seed(D)
    x = torch.zeros(4, 2, D + pad, dtype=BF, device="cuda")
    x[0, :, 5], x[1] = size, size
    x[2:] = (torch.rand(2, 2, D + pad, generator=g, device="cuda") * size).to(BF)
    x[2:, :, 7] = size
    x = x[..., :D]
    gain = (1 + 0.3 * torch.randn(D, generator=g, device="cuda")).to(BF)
    freqs, pos = binding.rope_freqs(D, 10000.0)[0], [0, 5, 77, 4000]
    out = torch.empty(4, 2, D, dtype=BF, device="cuda")
    binding.norm_rope(x, None, i32(pos), freqs.cuda(), gain, None, 0.0, out, None)
    for t in range(4):
        row = x[t].double().cpu().numpy()
        want = orc.norm_rotate(row, gain.double().cpu().numpy(), 0.0, pos[t], freqs.numpy())
        d = 4e-6 * np.abs(orc.norm_rotate(row, gain.double().cpu().numpy(), 0.0, 0, [])).max(-1, keepdims=True)
        assert (np.abs(out[t].double().cpu().numpy() - want) <= d + 2.0 ** -8 * (np.abs(want) + d)).all()
    assert binding.last_device_status() == 0
