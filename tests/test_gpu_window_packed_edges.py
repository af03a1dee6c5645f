"""Windowed and packed attention at their edges, in every form that a call may take.

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
