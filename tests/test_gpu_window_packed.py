"""Attention through a window and over a cache in 4 bits, on the device, against the fp64 definitions.

Tolerances of attention are those of the calls over 16 bits (test_gpu_attention.py): what a packed cache stands for goes to the
products exactly.  What the append writes and what is read back are compared byte by byte and bit by bit."""
import numpy as np
import pytest
import torch

from oracle import window_packed_oracle as orc
from paper_2509_15148_b200 import binding
from tests.test_gpu_attention import BF, FP, Batch, i32

pytestmark = pytest.mark.gpu


def pack_pool(x):
    """[pages, page, heads, D] -> what a packed cache of these values holds, [pages, heads, bytes] on the device, and its values in
    fp64; by the definition, whole arrays at a time (test_pool_of_the_tests_is_the_oracles checks it against the oracle's)."""
    pages, page, heads, D = x.shape
    g = x.double().cpu().numpy().transpose(0, 2, 1, 3).reshape(pages, heads, page, D // 32, 32)
    fine = np.isfinite(g).all(-1)
    g = np.where(fine[..., None], g, 0.0)
    scales = np.array([orc.scale_of(b) for b in range(209)])
    top = np.minimum(np.abs(g).max(-1) / 7, 2048.0).astype(np.float16).astype(np.float64)
    up = np.clip(np.searchsorted(scales, top), 1, 208)
    low, high = top - scales[up - 1], scales[up] - top
    byte = np.where((low < high) | ((low == high) & (up % 2 == 1)), up - 1, up)
    s = scales[byte][..., None]
    code = np.where(s > 0, np.clip(np.round(g / np.where(s > 0, s, 1.0)), -7, 7), 0).astype(np.int64)
    value = np.where(fine[..., None], code * s, np.nan).reshape(pages, heads, page, D).transpose(0, 2, 1, 3)
    byte = np.where(fine, byte, 255)
    n = (code + 8).reshape(pages, heads, page, D // 8, 8)
    word = sum(n[..., j] << (4 * (j // 2) + 16 * (j % 2)) for j in range(8)).astype(np.uint32)
    codes = np.ascontiguousarray(word).view(np.uint8).reshape(pages, heads, page // 8, 4 * D)
    pool = np.concatenate([codes, byte.astype(np.uint8).reshape(pages, heads, page // 8, D // 4)], -1).reshape(pages, heads, -1)
    return torch.from_numpy(pool).cuda(), torch.from_numpy(value).cuda()


def test_pool_of_the_tests_is_the_oracles():
    x = torch.randn(2, 16, 1, 64, generator=torch.Generator().manual_seed(0)).half()
    x[0, 3, 0, :32] *= 1e-5
    x[1, 2, 0, 5] = float("inf")
    pool, value = pack_pool(x)
    for p in range(2):
        block = pool[p, 0].cpu().numpy()
        assert np.array_equal(orc.unpack(block, 16, 64), value[p, :, 0].cpu().numpy(), equal_nan=True)
        for e in range(16):
            codes, scales = orc.packed_slot(x[p, e, 0].double().numpy())
            c0, s0 = orc.slot_bytes(e, 64)
            assert np.array_equal(block[c0:c0 + 32], codes) and np.array_equal(block[s0:s0 + 2], scales)


class Windowed(Batch):
    """A batch whose rows see through a window (0: everything), over a 16-bit or a packed cache."""

    def __init__(self, *args, window=0, sinks=0, packed=False, **kw):
        super().__init__(*args, **kw)
        self.window, self.sinks, self.packed = window, sinks, packed
        self.depth = None if self.pre is None else binding.tree_plan(self.parent, self.cu_h)[2].cuda()
        if packed:
            pools = []
            for name in ("k", "v"):
                pool, value = pack_pool(getattr(self, name))
                pools.append(pool)
                setattr(self, name, value)
            self.pools = pools
            self.handle = binding.PackedCache(*pools, self.table, self.page, self.D)

    def call(self, slack=(0, 0), out=None, q=None, lse=True, ws=None):
        mt, ml = self.mt + slack[0], self.ml + slack[1]
        name = "packed" if self.packed else "window"
        if ws is None:
            n = getattr(binding, name + "_attention_workspace_bytes")(self.B, self.M, self.Hq, self.Hk, self.D, mt, ml, self.window, self.sinks)
            ws = torch.full((n,), 255, dtype=torch.uint8, device="cuda")
        out = torch.full((self.M, self.Hq, self.D), float("nan"), dtype=self.dtype, device="cuda") if out is None else out
        l = torch.full((self.M, self.Hq), float("nan"), device="cuda") if lse else None
        getattr(binding, name + "_attention")(self.q if q is None else q, self.handle if self.packed else self.cache, self.ctx, self.cu, self.pre, self.end, self.depth,
                                              self.window, self.sinks, mt, ml, self.scale, out, l, ws)
        return out, l

    def see(self, b):
        """Truth values [tokens, slots] of sequence b, tokens at a time."""
        c, par = int(self.ctx_h[b]), self.parent[self.cu_h[b]:self.cu_h[b + 1]]
        n = len(par)
        tree, depth = np.zeros((n, n), bool), np.zeros(n, np.int64)
        for t in range(n):
            if par[t] == -2:
                continue
            if par[t] >= 0:
                tree[t], depth[t] = tree[par[t]], depth[par[t]] + 1
            tree[t, t] = True
        see = np.concatenate([np.repeat((par != -2)[:, None], c, 1), tree], 1)
        if self.window:
            place = np.concatenate([np.arange(c), c + depth])
            see &= (place[None] > (c + depth)[:, None] - self.window) | (place < self.sinks)[None]
        return see

    def dense(self):
        G = self.Hq // self.Hk
        out = torch.zeros(self.M, self.Hq, self.D, dtype=torch.float64, device="cuda")
        lse = torch.full((self.M, self.Hq), -float("inf"), dtype=torch.float64, device="cuda")
        for b in range(self.B):
            S = int(self.len_h[b])
            if self.tokens[b] == 0:
                continue
            see = torch.from_numpy(self.see(b)).cuda()
            pages = self.table[b, :-(-S // self.page)].long()
            rows = slice(int(self.cu_h[b]), int(self.cu_h[b + 1]))
            for h in range(self.Hk):
                k, v = (x[pages, :, h].flatten(0, 1)[:S].double() for x in (self.k, self.v))
                s = torch.einsum("tgd,sd->tgs", self.q[rows, h * G:(h + 1) * G].double(), torch.nan_to_num(k)) * self.scale
                s.masked_fill_(~see[:, None], -float("inf"))
                l = torch.logsumexp(s, -1)
                out[rows, h * G:(h + 1) * G] = torch.exp(s - torch.where(torch.isinf(l), 0.0, l)[..., None]) @ torch.nan_to_num(v)
                lse[rows, h * G:(h + 1) * G] = l
        return out, lse


def run(*args, **kw):
    b = Windowed(5, *args, **kw)
    out, lse = b.call()
    b.check(out, lse, *b.dense())
    assert binding.last_device_status() == 0
    return b, out, lse


def test_seen_by_the_tests_is_the_oracles():
    b = Windowed(1, [9, 4], [30, 2], 2, 1, 64, 8, BF, "random", 0.2, window=5, sinks=3)
    for i in range(2):
        assert np.array_equal(b.see(i), orc.sees(b.parent[b.cu_h[i]:b.cu_h[i + 1]], int(b.ctx_h[i]), 5, 3))


SMALL = [  # tokens, ctx, Hq, Hk, D, page, dtype, tree, padding
    ([1], [0], 4, 4, 64, 16, BF, "chain", 0.0),
    ([1], [1], 8, 1, 128, 8, FP, "chain", 0.0),
    ([3, 0, 1], [5, 9, 0], 6, 2, 64, 8, BF, "random", 0.0),
    ([7, 2], [40, 127], 5, 1, 128, 16, BF, "random", 0.3),
    ([20], [130], 14, 2, 128, 32, FP, "random", 0.2),
    ([9, 9, 9], [0, 128, 255], 8, 8, 64, 64, FP, "fan", 0.0),
    ([2], [256], 128, 1, 128, 128, BF, "random", 0.0),
    ([4, 30], [700, 300], 8, 2, 128, 256, FP, "random", 0.1),
]


@pytest.mark.parametrize("window, sinks", [(1, 0), (1, 3), (20, 0), (128, 4), (129, 130), (5000, 1)])
@pytest.mark.parametrize("case", SMALL)
def test_window(case, window, sinks):
    run(*case, window=window, sinks=sinks)


LARGE = [
    ([1] * 9, [126, 127, 128, 129, 254, 255, 256, 511, 1000], 32, 8, 128, 16, BF, "chain", 0.0),
    ([1] * 5, [4095, 1, 2047, 640, 63], 28, 4, 64, 64, FP, "chain", 0.0),
    ([1, 2], [70000, 33], 16, 2, 128, 128, BF, "random", 0.0),
    ([64], [20000], 8, 8, 128, 16, FP, "random", 0.1),
    ([24, 11, 17, 1, 24], [2500, 1733, 2048, 0, 300], 40, 8, 128, 16, BF, "random", 0.0),
    ([300, 7], [500, 4000], 12, 1, 64, 32, BF, "fan", 0.0),
    ([600], [1], 8, 2, 128, 16, FP, "chain", 0.0),
]


@pytest.mark.parametrize("window, sinks", [(1, 1), (200, 4), (512, 0), (2047, 300), (1 << 30, 0)])
@pytest.mark.parametrize("case", LARGE)
def test_window_over_longer_caches(case, window, sinks):
    run(*case, window=window, sinks=sinks)


def test_window_of_many_short_sequences():
    run([1] * 300, [1500 + i for i in range(300)], 8, 1, 128, 16, BF, "chain", 0.0, window=100, sinks=2)


def test_everything_within_the_window_is_attention_without_one():
    b, out, lse = run([24, 3], [900, 50], 8, 2, 128, 16, BF, "random", 0.1, window=4000, sinks=0)
    want, want_lse = b.attend()
    b.check(out, lse, want.double(), want_lse.double())


@pytest.mark.parametrize("packed", [False, True])
def test_pages_behind_the_window_may_be_gone(packed):
    """Freed pages (-1 in the table) of slots that nobody sees: not read, not flagged, although some share a tile with slots that are seen."""
    b = Windowed(3, [5, 1], [1000, 640], 8, 2, 128, 16, FP, "random", 0.0, window=100, sinks=20, packed=packed)
    want = b.dense()
    for i in range(2):
        gone = [c for c in range(b.table.shape[1]) if 20 <= 16 * c and 16 * c + 15 < int(b.ctx_h[i]) - 100 + 1]
        b.table[i, gone] = -1
        assert len(gone) > 30
    out, lse = b.call()
    b.check(out, lse, *want)
    assert binding.last_device_status() == 0
    b.table[0, int(b.ctx_h[0]) // 16 - 2] = -1       # one that is seen
    b.call()
    assert binding.last_device_status() == binding.DEV_PAGE_RANGE


def test_lengths_that_do_not_fit_are_flagged_and_depths_out_of_range_do_no_harm():
    b = Windowed(3, [5, 5], [300, 40], 8, 2, 64, 16, BF, "random", 0.0, window=50, sinks=2)
    want = b.dense()
    b.depth[5:] = torch.tensor([-(1 << 31), (1 << 31) - 1, 1 << 30, -5, 77], dtype=torch.int32)
    out, lse = b.call()
    assert (out[:5].double() - want[0][:5]).abs().max() <= 0.05 and binding.last_device_status() == 0
    b.ctx = i32([300, -1])
    out, lse = b.call()
    assert torch.isnan(out[5:]).all() and binding.last_device_status() == binding.DEV_SEQ_RANGE


# ---- the cache in 4 bits ----------------------------------------------------------------------------------------------
@pytest.mark.parametrize("D, dtype, heads, page, pad", [(64, BF, 2, 8, 0), (128, FP, 8, 16, 0), (128, BF, 1, 64, 8), (192, FP, 3, 16, 0), (256, BF, 2, 32, 0),
                                                        (64, FP, 5, 16, 3), (128, BF, 2, 16, 1)])
def test_append_writes_the_format_to_the_byte_and_is_read_back(D, dtype, heads, page, pad):
    rs = np.random.RandomState(3)
    g = torch.Generator(device="cuda").manual_seed(3)
    tokens, ctx = np.array([1, 0, 37, 200]), np.array([5, 3, 0, 8 * page - 3])
    M, B = int(tokens.sum()), 4
    k, v = ((torch.randn(M, heads, D + pad, generator=g, device="cuda") * 2).to(dtype)[..., :D] for _ in range(2))
    # magnitudes of every size, ties, zeros, what is not finite, what is too large
    k.mul_(torch.exp2(torch.randint(-16, 11, (M, heads, 1), generator=g, device="cuda").float()).to(dtype))
    v[3], v[4, 0, 3], v[5, 0, 40], v[6, -1, 7] = 0, float("nan"), float("inf"), 30000.0
    v[7, 0, :32] = torch.arange(-16, 16).to(dtype) / 2
    v[7, 0, 31] = 7.0
    v[8, 0, :32] = 2.0 ** -14 * torch.arange(32).to(dtype) / 32
    need = -(-(tokens + ctx) // page)
    n = int(need.sum()) + 2
    perm, tab, at = rs.permutation(n), np.full((B, int(need.max())), -1), 0
    for b in range(B):
        tab[b, :need[b]] = perm[at:at + need[b]]
        at += need[b]
    block = binding.packed_block_bytes(page, D)
    pools = [torch.full((n, heads, block), 0xAA, dtype=torch.uint8, device="cuda") for _ in range(2)]
    cache = binding.PackedCache(*pools, i32(tab), page, D)
    cu = np.concatenate([[0], np.cumsum(tokens)])
    binding.packed_append(k, v, cache, i32(ctx), i32(cu), 200)
    # the same by the definition
    dst = [torch.full((n, page, heads, D), 5.0, dtype=dtype, device="cuda") for _ in range(2)]
    binding.packed_read(cache, i32(ctx + tokens), int((ctx + tokens).max()), binding.PagedCache(*dst, i32(tab)))
    assert binding.last_device_status() == 0
    seq = np.searchsorted(cu, np.arange(M), side="right") - 1
    slot = ctx[seq] + np.arange(M) - cu[seq]
    pages, offs = tab[seq, slot // page], slot % page
    for new, pool, back in zip((k, v), pools, dst):
        x = torch.zeros(n, page, heads, D, dtype=dtype, device="cuda")
        x[torch.as_tensor(pages).cuda(), torch.as_tensor(offs).cuda()] = new
        want, value = pack_pool(x)
        mask = np.zeros((n, 1, block), bool)
        for p, o in zip(pages, offs):
            c0, s0 = orc.slot_bytes(int(o), D)
            mask[p, 0, c0:c0 + D // 2] = mask[p, 0, s0:s0 + D // 32] = True
        mask = torch.from_numpy(mask).cuda()
        assert torch.equal(pool, torch.where(mask, want, torch.tensor(0xAA, dtype=torch.uint8, device="cuda")))
        got = back[torch.as_tensor(pages).cuda(), torch.as_tensor(offs).cuda()].double()
        assert torch.equal(torch.nan_to_num(got, 1e30), torch.nan_to_num(value[torch.as_tensor(pages).cuda(), torch.as_tensor(offs).cuda()], 1e30))
        dead = np.ones((n, page), bool)
        for b in range(B):
            s = np.arange(ctx[b] + tokens[b])
            dead[tab[b, s // page], s % page] = False
        assert (back[torch.from_numpy(dead).cuda()] == 5).all()        # slots behind the lengths as they were


def test_read_back_in_the_other_type_and_through_other_strides():
    x = (torch.randn(6, 16, 2, 128, generator=torch.Generator().manual_seed(1)) * 3).bfloat16()
    pool, value = pack_pool(x)
    wide = torch.full((6, 4, pool.shape[2] + 32), 0, dtype=torch.uint8, device="cuda")
    wide[:, ::2, :-32] = pool
    src = binding.PackedCache(wide[:, ::2, :-32], wide[:, ::2, :-32], i32([[3, 1, 5], [0, 2, 4]]), 16, 128)
    back = torch.zeros(6, 2, 16, 128, dtype=FP, device="cuda").transpose(1, 2)
    back2 = torch.zeros_like(back, memory_format=torch.preserve_format)
    binding.packed_read(src, i32([48, 20]), 48, binding.PagedCache(back, back2, i32([[0, 1, 2], [3, 4, 5]])))
    for i, p in enumerate([3, 1, 5, 0]):
        assert torch.equal(back[i].double(), value[p]) and torch.equal(back2[i].double(), value[p])
    assert torch.equal(back[4, :4].double(), value[2, :4]) and (back[4, 4:] == 0).all() and (back[5] == 0).all()
    assert binding.last_device_status() == 0
    binding.packed_read(src, i32([48, 60]), 48, binding.PagedCache(back, back2, i32([[0, 1, 2], [3, 4, 6]])))
    assert binding.last_device_status() == binding.DEV_SEQ_RANGE | binding.DEV_PAGE_RANGE
    binding.packed_read(src, i32([-3, 0]), 0, binding.PagedCache(back, back2, i32([[0, 1, 2], [3, 4, 5]])))
    assert binding.last_device_status() == 0


def test_append_flags_bad_pages_and_lengths():
    k = torch.randn(4, 1, 64, device="cuda").bfloat16()
    pool = torch.full((2, 1, binding.packed_block_bytes(8, 64)), 7, dtype=torch.uint8, device="cuda")
    for table, ctx, mt, bits in (([[0], [2]], [0, 0], 2, binding.DEV_PAGE_RANGE), ([[0], [-1]], [0, 0], 2, binding.DEV_PAGE_RANGE), ([[0], [1]], [0, 7], 2, binding.DEV_PAGE_RANGE),
                                 ([[0], [1]], [0, -1], 2, binding.DEV_SEQ_RANGE), ([[0], [1]], [0, 0], 1, binding.DEV_SEQ_RANGE)):
        c = binding.PackedCache(pool, pool.clone(), i32(table), 8, 64)
        binding.packed_append(k, k, c, i32(ctx), i32([0, 1, 4] if mt == 1 else [0, 2, 4]), mt)
        assert binding.last_device_status() == bits


@pytest.mark.parametrize("case", SMALL)
def test_packed(case):
    run(*case, packed=True)


@pytest.mark.parametrize("window, sinks", [(1, 0), (20, 3), (129, 130)])
@pytest.mark.parametrize("case", SMALL[2:])
def test_packed_through_a_window(case, window, sinks):
    run(*case, window=window, sinks=sinks, packed=True)


@pytest.mark.parametrize("case", LARGE)
def test_packed_over_longer_caches(case):
    run(*case, packed=True)


@pytest.mark.parametrize("window, sinks", [(200, 4), (2047, 300)])
@pytest.mark.parametrize("case", LARGE)
def test_packed_over_longer_caches_through_a_window(case, window, sinks):
    run(*case, window=window, sinks=sinks, packed=True)


FEW = [  # numbers of rows at and around what a form for few rows takes
    ([1, 0, 1], [4000, 5, 129], 8, 1, 64, 16, BF, "chain", 0.0),
    ([2, 1], [1300, 126], 16, 2, 128, 8, FP, "random", 0.0),
    ([3, 3], [513, 128], 6, 2, 128, 16, BF, "random", 0.0),
    ([5], [20000], 12, 2, 64, 64, FP, "random", 0.2),
    ([8, 2], [900, 30], 16, 4, 128, 32, BF, "random", 0.1),
    ([11, 1, 0], [3000, 0, 7], 12, 4, 128, 128, FP, "random", 0.1),
    ([17, 40], [700, 260], 2, 2, 64, 16, BF, "fan", 0.0),
    ([16], [300], 32, 8, 128, 256, BF, "chain", 0.0),
    ([65], [140], 2, 2, 128, 16, BF, "random", 0.1),
    ([6] * 40, [100 + 9 * i for i in range(40)], 24, 4, 128, 16, FP, "random", 0.1),
]


@pytest.mark.parametrize("window, sinks", [(0, 0), (1, 2), (150, 4), (1000, 0)])
@pytest.mark.parametrize("case", FEW)
def test_packed_with_few_rows(case, window, sinks):
    run(*case, window=window, sinks=sinks, packed=True)


def test_packed_with_large_pages_loose_bounds_and_scattered_rows():
    b = Windowed(5, [11, 30], [5000, 700], 8, 2, 128, 512, BF, "random", 0.1, packed=True)
    want = b.dense()
    b.check(*b.call(slack=(20, 9000)), *want)
    wide = torch.zeros(b.M, 2 * b.Hq, 2 * b.D, dtype=BF, device="cuda")
    wide[:, ::2, :b.D] = b.q
    out = torch.zeros(b.M, b.Hq, b.D + 8, dtype=BF, device="cuda")[..., :b.D]
    b.check(*b.call(q=wide[:, ::2, :b.D], out=out), *want)
    b.check(b.call(lse=False)[0], None, want[0], want[1])
    assert binding.last_device_status() == 0


def test_packed_pages_that_are_missing_read_as_zeros():
    b = Windowed(5, [3], [400], 4, 1, 128, 16, FP, "random", 0.0, packed=True)
    b.k[b.table[0, 5].item()], b.v[b.table[0, 5].item()] = 0, 0
    b.k[b.table[0, 11].item()], b.v[b.table[0, 11].item()] = 0, 0
    want = b.dense()
    b.table[0, 5], b.table[0, 11] = b.n_pages, -7
    out, lse = b.call()
    b.check(out, lse, *want)
    assert binding.last_device_status() == binding.DEV_PAGE_RANGE


def test_nan_in_a_packed_key_reaches_the_rows_that_see_it():
    b = Windowed(5, [3], [300], 4, 1, 128, 16, BF, "chain", 0.0, packed=True)
    b.pools[0][b.table[0, 300 // 16].item(), 0, orc.slot_bytes((300 + 1) % 16, 128)[1]] = 255      # key of the second drafted token
    out, lse = b.call()
    assert torch.isnan(lse[1:]).all() and torch.isnan(out[1:]).all() and not torch.isnan(lse[0]).any() and not torch.isnan(out[0]).any()


@pytest.mark.parametrize("packed", [False, True])
def test_results_do_not_depend_on_what_the_workspace_held_and_repeat(packed):
    b = Windowed(5, [13], [40000], 8, 2, 128, 64, BF, "random", 0.0, window=30000, sinks=4, packed=packed)
    first = b.call()
    again = b.call(ws=torch.zeros(1 << 26, dtype=torch.uint8, device="cuda"))
    assert torch.equal(first[0], again[0]) and torch.equal(first[1], again[1])


def test_captured_replayed_and_on_another_stream():
    """Two graphs with workspaces of their own, the append and both attentions in each, replayed in turn on other streams."""
    made = []
    for seed in (5, 6):
        b = Windowed(seed, [5, 9], [900, 40], 8, 2, 128, 16, BF, "random", 0.0, window=300, sinks=4, packed=True)
        w = Windowed(seed, [5, 9], [900, 40], 8, 2, 128, 16, BF, "random", 0.0, window=300, sinks=4)
        n = binding.packed_attention_workspace_bytes(b.B, b.M, b.Hq, b.Hk, b.D, b.mt, b.ml, 300, 4)
        n2 = binding.window_attention_workspace_bytes(b.B, b.M, b.Hq, b.Hk, b.D, b.mt, b.ml, 300, 4)
        ws, ws2 = (torch.empty(x, dtype=torch.uint8, device="cuda") for x in (n, n2))
        new = torch.randn(2, b.M, b.Hk, b.D, device="cuda").bfloat16()
        at = np.concatenate([b.ctx_h[i] + np.arange(b.tokens[i]) for i in range(b.B)])
        seq = np.repeat(np.arange(b.B), b.tokens)
        page, off = torch.as_tensor(b.table_h[seq, at // 16]).cuda(), torch.as_tensor(at % 16).cuda()
        side = torch.cuda.Stream()
        out, out2 = torch.empty(b.M, b.Hq, b.D, dtype=BF, device="cuda"), torch.empty(b.M, b.Hq, b.D, dtype=BF, device="cuda")

        def step():
            binding.packed_append(new[0], new[1], b.handle, b.ctx, b.cu, b.mt)
            l = b.call(out=out, ws=ws)[1]
            return l, w.call(out=out2, ws=ws2)[1]
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            step()
        torch.cuda.current_stream().wait_stream(side)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            lse, lse2 = step()
        made.append((b, w, new, page, off, graph, out, out2, lse, lse2, side, step))
    for turn in range(2):
        for b, w, new, page, off, graph, out, out2, lse, lse2, side, _ in made:
            new.normal_()
            out.fill_(float("nan"))
            out2.fill_(float("nan"))
            side.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(side):
                graph.replay()
        torch.cuda.synchronize()
        for b, w, new, page, off, graph, out, out2, lse, lse2, side, _ in made:
            for i, x in enumerate((b.k, b.v)):
                x[page, off] = pack_pool(new[i][:, None].repeat(1, 8, 1, 1))[1][:, 0]
            b.check(out, lse, *b.dense())
            w.check(out2, lse2, *w.dense())
    assert binding.last_device_status() == 0


@pytest.mark.parametrize("packed", [False, True])
@pytest.mark.parametrize("tokens, ctx", [([2], [300]), ([400], [300]), ([2], [60000])])
def test_waits_that_run_out_are_reported(tokens, ctx, packed):
    b = Windowed(5, tokens, ctx, 8, 2, 128, 16, BF, "chain", 0.0, window=50000, sinks=0, packed=packed)
    binding.debug_set_wait(2_000_000, True)
    try:
        b.call()
        with pytest.raises(binding.AttsError) as e:
            binding.last_device_status()
        assert e.value.status == 9
    finally:
        binding.debug_set_wait(0, False)
    b.check(*b.call(), *b.dense())
    assert binding.last_device_status() == 0


@pytest.mark.parametrize("packed", [False, True])
def test_empty_batches_and_sizes_that_a_workspace_does_not_fit(packed):
    b = Windowed(5, [0, 0], [5, 0], 4, 2, 64, 8, BF, "chain", 0.0, window=5, packed=packed)
    b.mt, b.ml = 0, 5
    assert b.call()[0].numel() == 0
    b = Windowed(5, [3], [40000], 4, 2, 64, 8, BF, "chain", 0.0, window=30000, packed=packed)
    with pytest.raises(binding.AttsError) as e:
        b.call(ws=torch.empty(256, dtype=torch.uint8, device="cuda"))
    assert e.value.status == 4 and binding.last_device_status() == 0


def test_norm_append_attend_and_read_back_as_a_layer_uses_them():
    """norm_rope -> packed_append -> packed_attention, three steps of drafted trees over one growing cache, against the definitions
    chained in fp64 on what each call was given."""
    rs, g = np.random.RandomState(9), torch.Generator(device="cuda").manual_seed(9)
    B, Hq, Hk, D, page, T = 3, 8, 2, 128, 16, 6
    pool = [torch.zeros(B * 4, Hk, binding.packed_block_bytes(page, D), dtype=torch.uint8, device="cuda") for _ in range(2)]
    table = rs.permutation(B * 4).reshape(B, 4)
    cache = binding.PackedCache(*pool, i32(table), page, D)
    freqs = binding.rope_freqs(D, 500000.0)[0].cuda()
    gain = (1 + 0.3 * torch.randn(2, D, generator=g, device="cuda")).to(BF)
    parent, cu = np.array([-1, 0, 1, 0, 3, -1] * B, np.int32), np.arange(B + 1) * T
    pre, end, depth = binding.tree_plan(parent, cu)
    held = [torch.zeros(B, 64, Hk, D, dtype=torch.float64) for _ in range(2)]
    for step in range(3):
        ctx = np.array([3 * step, 4 * step, 10 + 2 * step])
        q, k, v = (torch.randn(B * T, h, D, generator=g, device="cuda").to(BF) for h in (Hq, Hk, Hk))
        pos = i32(np.repeat(ctx, T) + depth.numpy())
        q2, k2 = torch.empty_like(q), torch.empty_like(k)
        binding.norm_rope(q, k, pos, freqs, gain[0], gain[1], EPS, q2, k2)
        binding.packed_append(k2, v, cache, i32(ctx), i32(cu), T)
        out, lse = torch.empty_like(q), torch.empty(B * T, Hq, device="cuda")
        ws = torch.empty(binding.packed_attention_workspace_bytes(B, B * T, Hq, Hk, D, T, 40, 7, 2), dtype=torch.uint8, device="cuda")
        binding.packed_attention(q2, cache, i32(ctx), i32(cu), pre.cuda(), end.cuda(), depth.cuda(), 7, 2, T, 40, D ** -0.5, out, lse, ws)
        for b in range(B):
            for i, x in enumerate((k2, v)):
                held[i][b, ctx[b]:ctx[b] + T] = pack_pool(x[b * T:(b + 1) * T][:, None].repeat(1, 8, 1, 1))[1][:, 0].cpu()
            see = torch.from_numpy(orc.sees(parent[:T], int(ctx[b]), 7, 2))
            n = see.shape[1]
            for h in range(Hq):
                s = (q2[b * T:(b + 1) * T, h].double().cpu() @ held[0][b, :n, h // 4].T) * D ** -0.5
                p = torch.softmax(s.masked_fill(~see, -float("inf")), -1)
                vv = held[1][b, :n, h // 4]
                err = (out[b * T:(b + 1) * T, h].double().cpu() - p @ vv).abs() - 2.0 ** -8 * (vv.abs().max() + (p @ vv).abs()) - 1e-4 * vv.abs().max()
                assert err.max() <= 0
    assert binding.last_device_status() == 0


def test_example_of_a_layer_whose_cache_stops_growing():
    """examples/packed_step.py, every step against the definitions on what the cache has to hold."""
    import importlib.util
    import os

    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "packed_step.py")
    spec = importlib.util.spec_from_file_location("packed_step", path)
    ex = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(ex)
    torch.manual_seed(3)
    B, line = 3, 9
    layer = ex.PackedLayer(samples=B, slots=256, pages=24, hidden=128, heads=4, kv_heads=2, head_dim=64, window=40, sinks=3)
    parent = list(range(-1, line - 1)) + [4, line]
    T = len(parent)
    held = [torch.zeros(B, 256, 2, 64, dtype=torch.float64) for _ in range(2)]
    for turn in range(16):
        ctx = layer.lens.tolist()
        _, q, k, v, out, lse = layer.step(torch.randn(B * T, 128, device="cuda").bfloat16(), parent * B, [T * b for b in range(B + 1)])
        for b in range(B):
            rows = slice(b * T, (b + 1) * T)
            for i, x in enumerate((k, v)):
                held[i][b, ctx[b]:ctx[b] + T] = pack_pool(x[rows][:, None].repeat(1, 8, 1, 1))[1][:, 0].cpu()
            see = torch.from_numpy(orc.sees(parent, ctx[b], 40, 3))
            n = see.shape[1]
            for h in range(4):
                kk, vv = held[0][b, :n, h // 2], held[1][b, :n, h // 2]
                s = ((q[rows, h].double().cpu() @ kk.T) * layer.scale).masked_fill(~see, -float("inf"))
                want = torch.softmax(s, -1) @ vv
                assert ((out[rows, h].double().cpu() - want).abs() <= 2.0 ** -8 * (vv.abs().max() + want.abs()) + 1e-4 * vv.abs().max()).all()
                want_lse = torch.logsumexp(s, -1)
                assert ((lse[rows, h].double().cpu() - want_lse).abs() <= 5e-5 + 1e-5 * want_lse.abs()).all()
        layer.lens += line
        layer.release()
    assert 24 - len(layer.free) <= B * 5 and binding.last_device_status() == 0


def test_append_and_read_back_of_more_heads_than_a_block_has_threads_for():
    """24 heads of 128 and 3 of 64: more channels a token than threads, and a number of threads that does not divide a block."""
    for heads, D in ((24, 128), (3, 64), (40, 256)):
        g = torch.Generator(device="cuda").manual_seed(heads)
        k, v = (torch.randn(70, heads, D, generator=g, device="cuda").half() for _ in range(2))
        pools = [torch.zeros(5, heads, binding.packed_block_bytes(16, D), dtype=torch.uint8, device="cuda") for _ in range(2)]
        cache = binding.PackedCache(*pools, i32([[4, 0, 2, 1, 3]]), 16, D)
        binding.packed_append(k, v, cache, i32([3]), i32([0, 70]), 70)
        back = [torch.zeros(5, 16, heads, D, dtype=FP, device="cuda") for _ in range(2)]
        binding.packed_read(cache, i32([73]), 80, binding.PagedCache(*back, i32([[4, 0, 2, 1, 3]])))
        for x, y in zip((k, v), back):
            want = pack_pool(x[:, None].repeat(1, 8, 1, 1))[1][:, 0]
            got = y[torch.tensor([4, 0, 2, 1, 3], device="cuda")].flatten(0, 1)[3:73].double()
            assert torch.equal(got, want)
    assert binding.last_device_status() == 0


@pytest.mark.parametrize("rows", [4, 40, 200])
def test_infinite_scores_and_values_reach_the_rows_that_see_them(rows):
    """+inf among a row's scores makes its out and lse NaN, as in the attention over 16 bits, in every form that takes a packed cache."""
    b = Windowed(5, [rows], [300], 2, 2, 64, 16, BF, "chain", 0.0, packed=True)
    b.q[1, 0, :] = float("inf")
    out, lse = b.call()
    assert torch.isnan(lse[1, 0]) and torch.isnan(out[1, 0]).all()
    assert not torch.isnan(lse[0]).any() and not torch.isnan(lse[2:]).any() and not torch.isnan(out[2:]).any()


EPS = 1e-6
