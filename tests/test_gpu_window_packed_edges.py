"""Windowed and packed attention at their edges, in every form that a call may take.

A call's form goes by the rows that a sequence's key head can have (drafted tokens times the query heads that share it): over a packed
cache up to 8 and up to 16, in both up to 64, up to 128, more; over 16 bits also many short sequences.  ROWS has a batch of each.
Tolerances are those of test_gpu_attention.py."""
import pytest

from paper_2509_15148_b200 import binding
from tests.test_gpu_attention import BF
from tests.test_gpu_window_packed import Windowed

pytestmark = pytest.mark.gpu

ROWS = {  # tokens of the longest sequence, Hq, Hk
    "8": (4, 4, 2), "16": (4, 8, 2), "64": (20, 4, 2), "128": (100, 2, 2), "more": (200, 4, 2),
}


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
