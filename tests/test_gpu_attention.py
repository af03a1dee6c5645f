"""Attention of drafted tokens over a paged cache, on the device, against the fp64 definitions.

Tolerances.  Probabilities are rounded to the inputs' type before they multiply v, and the output once more: with u the
type's unit roundoff (2^-8 bf16, 2^-11 fp16) an output is off by at most u (sum p |v| + |o|) <= u (max |v| + |o|), and 1e-4
max |v| covers the fp32 part (scores of magnitude up to 40 off by 2e-5, exponentials and sums by 1e-5).  lse: the same 2e-5
on a score and 1e-5 on a sum: 5e-5 + 1e-5 |lse|.  A weight is a sum of exponentials, each off by 1e-4 of itself: 1e-4 w."""
import numpy as np
import pytest
import torch

from oracle import attention_oracle as orc
from paper_2509_15148_b200 import binding
from tests.test_attention_plan import random_parents

pytestmark = pytest.mark.gpu

BF, FP = torch.bfloat16, torch.float16
UNIT = {BF: 2.0 ** -8, FP: 2.0 ** -11}   # half a step of 8 and 11 significant bits, relative


def i32(x):
    return torch.as_tensor(np.asarray(x), dtype=torch.int32).cuda()


class Batch:
    """A cache, its table, drafted rows and their trees; dead slots and unused pages hold NaN."""

    def __init__(self, seed, tokens, ctx, Hq, Hk, D, page, dtype, tree="random", pad=0.0, layout="nhd", qscale=1.0, spare=3):
        rs = np.random.RandomState(seed)
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.tokens, self.ctx_h = np.array(tokens), np.array(ctx)
        self.B, self.M, self.Hq, self.Hk, self.D, self.page, self.dtype = len(tokens), int(sum(tokens)), Hq, Hk, D, page, dtype
        self.cu_h = np.concatenate([[0], np.cumsum(tokens)])
        self.len_h = self.tokens + self.ctx_h
        need = -(-self.len_h // page)
        self.n_pages = int(need.sum()) + spare
        perm = rs.permutation(self.n_pages)
        self.table_h = np.full((self.B, max(1, int(need.max()))), 0, np.int64)
        at = 0
        for b in range(self.B):
            self.table_h[b, :need[b]] = perm[at:at + need[b]]
            at += need[b]
        shape = (self.n_pages, page, Hk, D) if layout == "nhd" else (self.n_pages, Hk, page, D)
        k, v = (torch.full(shape, float("nan"), device="cuda", dtype=dtype) for _ in range(2))
        self.k, self.v = (k, v) if layout == "nhd" else (k.transpose(1, 2), v.transpose(1, 2))
        for b in range(self.B):
            for j in range(need[b]):
                n = min(page, int(self.len_h[b]) - j * page)
                for c in (self.k, self.v):
                    c[self.table_h[b, j], :n] = torch.randn(n, Hk, D, generator=g, device="cuda").to(dtype)
        self.q = (torch.randn(self.M, Hq, D, generator=g, device="cuda") * qscale).to(dtype)
        par = []
        for t in tokens:
            if tree == "chain":
                par.append(np.arange(-1, t - 1))
            elif tree == "fan":
                each = max(1, -(-t // 4))
                i = np.arange(t)
                par.append(np.where(i % each == 0, -1, i - 1))
            else:
                par.append(random_parents(rs, t, pad))
        self.parent = np.concatenate(par).astype(np.int32) if par else np.zeros(0, np.int32)
        if tree == "chain":
            self.pre = self.end = None
        else:
            self.pre, self.end = (x.cuda() for x in binding.tree_plan(self.parent, self.cu_h)[:2])
        self.table, self.ctx, self.cu = i32(self.table_h), i32(ctx), i32(self.cu_h)
        self.cache = binding.PagedCache(self.k, self.v, self.table)
        self.mt, self.ml = int(self.tokens.max()), int(self.len_h.max())
        self.scale = D ** -0.5

    def attend(self, slack=(0, 0), out=None, q=None, lse=True):
        mt, ml = self.mt + slack[0], self.ml + slack[1]
        ws = torch.full((binding.tree_attention_workspace_bytes(self.B, self.M, self.Hq, self.Hk, self.D, mt, ml),), 255,
                        dtype=torch.uint8, device="cuda")
        out = torch.full((self.M, self.Hq, self.D), float("nan"), dtype=self.dtype, device="cuda") if out is None else out
        l = torch.full((self.M, self.Hq), float("nan"), device="cuda") if lse else None
        binding.tree_attention(self.q if q is None else q, self.cache, self.ctx, self.cu, self.pre, self.end, mt, ml, self.scale, out, l, ws)
        return out, l

    def weights(self, lse, win=None, slack=(0, 0), cols=None):
        mt, ml = self.mt + slack[0], self.ml + slack[1]
        out = torch.full((self.B, self.Hk, cols or ml), float("nan"), device="cuda")
        binding.cache_weights(self.q, self.cache, lse, self.ctx, self.cu, self.pre, self.end, mt, ml, self.scale, win, out)
        return out

    def dense(self):
        """The definition in fp64 on the device, whole sequences at a time: (out, lse, weights)."""
        G = self.Hq // self.Hk
        out = torch.zeros(self.M, self.Hq, self.D, dtype=torch.float64, device="cuda")
        lse = torch.full((self.M, self.Hq), -float("inf"), dtype=torch.float64, device="cuda")
        w = torch.zeros(self.B, self.Hk, self.ml, dtype=torch.float64, device="cuda")
        for b in range(self.B):
            n, S, c = int(self.tokens[b]), int(self.len_h[b]), int(self.ctx_h[b])
            if n == 0:
                continue
            par = self.parent[self.cu_h[b]:self.cu_h[b + 1]]
            see = np.zeros((n, S), bool)
            for t in range(n):
                if par[t] == -2:
                    continue
                see[t, :c] = True
                if par[t] >= 0:
                    see[t, c:] = see[par[t], c:]
                see[t, c + t] = True
            see = torch.from_numpy(see).cuda()
            pages = self.table[b, :-(-S // self.page)].long()
            rows = slice(int(self.cu_h[b]), int(self.cu_h[b + 1]))
            for h in range(self.Hk):
                k, v = (x[pages, :, h].flatten(0, 1)[:S].double() for x in (self.k, self.v))
                q = self.q[rows, h * G:(h + 1) * G].double()
                s = torch.einsum("tgd,sd->tgs", q, k) * self.scale
                s.masked_fill_(~see[:, None], -float("inf"))
                l = torch.logsumexp(s, -1)
                p = torch.exp(s - torch.where(torch.isinf(l), 0.0, l)[..., None])
                out[rows, h * G:(h + 1) * G] = p @ v
                lse[rows, h * G:(h + 1) * G] = l
                w[b, h, :S] = p.sum((0, 1))
        return out, lse, w

    def check(self, out, lse, want_out, want_lse):
        u = UNIT[self.dtype]
        vmax = torch.nan_to_num(self.v.float()).abs().max().item()
        err = (out.double() - want_out).abs() - u * (vmax + want_out.abs()) - 1e-4 * vmax
        assert not torch.isnan(out).any() and err.max().item() <= 0, err.max().item()
        if lse is not None:
            dead = torch.isinf(want_lse)
            assert torch.equal(torch.isinf(lse), dead) and (lse[dead] < 0).all()
            e = (lse.double() - want_lse)[~dead].abs() - 5e-5 - 1e-5 * want_lse[~dead].abs()
            assert not torch.isnan(lse).any() and (e.numel() == 0 or e.max().item() <= 0), e.max().item()

    def check_weights(self, got, want):
        e = (got[..., :self.ml].double() - want).abs() - 1e-4 * want.abs() - 1e-9
        assert not torch.isnan(got).any() and e.max().item() <= 0, e.max().item()


SMALL = [  # tokens, ctx, Hq, Hk, D, page, dtype, tree, padding
    ([1], [0], 4, 4, 64, 16, BF, "chain", 0.0),
    ([1], [1], 8, 1, 128, 8, FP, "chain", 0.0),
    ([3, 0, 1], [5, 9, 0], 6, 2, 64, 8, BF, "random", 0.0),
    ([7, 2], [40, 127], 5, 1, 128, 16, BF, "random", 0.3),
    ([20], [130], 14, 2, 128, 32, FP, "random", 0.2),
    ([9, 9, 9], [0, 128, 255], 8, 8, 64, 64, FP, "fan", 0.0),
    ([2], [256], 128, 1, 128, 128, BF, "random", 0.0),
]


@pytest.mark.parametrize("case", SMALL)
def test_attention_and_weights_against_the_oracle(case):
    tokens, ctx, Hq, Hk, D, page, dtype, tree, pad = case
    b = Batch(5, tokens, ctx, Hq, Hk, D, page, dtype, tree, pad)
    host = [x.double().cpu().numpy() for x in (b.q, b.k, b.v)]
    want_out, want_lse = orc.tree_attention(*host, b.table_h, b.ctx_h, b.cu_h, b.parent, b.scale)
    out, lse = b.attend()
    b.check(out, lse, torch.from_numpy(want_out).cuda(), torch.from_numpy(want_lse).cuda())
    w = b.weights(torch.from_numpy(want_lse).float().cuda())
    lse32 = want_lse.astype(np.float32).astype(np.float64)
    b.check_weights(w, torch.from_numpy(orc.cache_weights(host[0], host[1], b.table_h, lse32, b.ctx_h, b.cu_h, b.parent, b.scale, b.ml)).cuda())
    assert binding.last_device_status() == 0


LARGE = [
    # one token over caches whose lengths sit at, before and behind the edges of pages and tiles
    ([1] * 9, [126, 127, 128, 129, 254, 255, 256, 511, 1000], 32, 8, 128, 16, BF, "chain", 0.0),
    ([1] * 5, [4095, 1, 2047, 640, 63], 28, 4, 64, 64, FP, "chain", 0.0),
    ([1, 2], [70000, 33], 16, 2, 128, 128, BF, "random", 0.0),          # one sequence far longer than the other
    ([64], [20000], 8, 8, 128, 16, FP, "random", 0.1),
    ([24, 11, 17, 1, 24], [2500, 1733, 2048, 0, 300], 40, 8, 128, 16, BF, "random", 0.0),
    ([33, 97], [700, 90], 14, 2, 64, 8, BF, "random", 0.2),
    ([600], [300], 40, 8, 128, 32, BF, "fan", 0.0),
    ([900, 411], [513, 0], 24, 8, 128, 64, FP, "fan", 0.0),
    ([700, 1, 350], [0, 777, 120], 16, 16, 64, 128, BF, "chain", 0.0),
    ([513], [1024], 64, 8, 128, 256, FP, "chain", 0.0),
    ([130, 260], [5, 6], 100, 1, 128, 4096, BF, "random", 0.1),
    ([300], [100], 9, 3, 128, 16, BF, "random", 0.5),
]


@pytest.mark.parametrize("case", LARGE)
def test_attention_and_weights_at_size(case):
    tokens, ctx, Hq, Hk, D, page, dtype, tree, pad = case
    b = Batch(6, tokens, ctx, Hq, Hk, D, page, dtype, tree, pad)
    out, lse = b.attend()
    want_out, want_lse, want_w = b.dense()
    b.check(out, lse, want_out, want_lse)
    # bounds that are not tight change the launch, not the answer
    out2, lse2 = b.attend(slack=(50, 900))
    b.check(out2, lse2, want_out, want_lse)
    b.check_weights(b.weights(want_lse.float()), want_w)
    assert binding.last_device_status() == 0


def test_results_repeat_bit_for_bit():
    b = Batch(7, [40, 9], [3000, 5000], 16, 4, 128, 16, BF)
    first = b.attend()
    w = b.weights(first[1])
    for _ in range(5):
        again = b.attend()
        assert torch.equal(first[0], again[0]) and torch.equal(first[1], again[1]) and torch.equal(w, b.weights(first[1]))


@pytest.mark.parametrize("layout", ["nhd", "hnd"])
def test_strided_rows_and_cache_layouts(layout):
    b = Batch(8, [30, 5], [200, 77], 12, 4, 128, 32, BF, layout=layout)
    want_out, want_lse, want_w = b.dense()
    wide = torch.full((b.M, b.Hq + 8, b.D + 8), float("nan"), dtype=b.dtype, device="cuda")
    wide[:, 4:4 + b.Hq, :b.D] = b.q
    host = torch.full((b.Hq, b.M + 1, b.D), float("nan"), dtype=b.dtype, device="cuda")
    out = host[:, :b.M].transpose(0, 1)
    b.attend(q=wide[:, 4:4 + b.Hq, :b.D], out=out, lse=False)
    b.check(out, None, want_out, want_lse)
    assert torch.isnan(host[:, b.M]).all()
    b.q = wide[:, 4:4 + b.Hq, :b.D]
    b.check_weights(b.weights(want_lse.float()), want_w)


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("qscale", [1e-3, 30.0])
def test_flat_and_peaked_rows(dtype, qscale):
    b = Batch(9, [50, 1], [900, 3000], 8, 2, 128, 16, dtype, qscale=qscale)
    b.scale = 0.08
    out, lse = b.attend()
    want_out, want_lse, _ = b.dense()
    # scores reach qscale * 30: their fp32 error grows with them (2^-22 of the sum of the products' magnitudes)
    extra = 4e-6 * qscale * 30
    vmax = torch.nan_to_num(b.v.float()).abs().max().item()
    assert ((out.double() - want_out).abs() <= UNIT[dtype] * (vmax + want_out.abs()) + (1e-4 + 2 * extra) * vmax).all()
    assert ((lse.double() - want_lse).abs() <= 5e-5 + extra + 1e-5 * want_lse.abs()).all()


def test_maximum_that_grows_along_the_cache():
    """Every later key scores higher, by up to hundreds: the running maximum moves at every tile."""
    b = Batch(10, [4], [2000], 4, 2, 128, 16, BF)
    b.q[:] = 0
    b.q[..., 0] = 8.0
    for s in range(2000):
        b.k[b.table_h[0, s // 16], s % 16, :, 0] = s / 8.0
    b.scale = 0.25
    out, lse = b.attend()
    want_out, want_lse, _ = b.dense()
    b.check(out, lse, want_out, want_lse)


@pytest.mark.parametrize("Hq,Hk,D,dtype,most", [(8, 2, 64, BF, 4), (16, 8, 128, BF, 2), (24, 4, 128, FP, 17), (7, 1, 64, FP, 40)])
def test_many_sequences_and_empty_ones(Hq, Hk, D, dtype, most):
    """More (sequence, head) pairs than SMs, each short, some without drafts."""
    rs = np.random.RandomState(11)
    tokens = rs.randint(0, most, 300)
    ctx = rs.randint(0, 200, 300)
    b = Batch(11, tokens, ctx, Hq, Hk, D, 16, dtype, pad=0.1)
    out, lse = b.attend()
    want_out, want_lse, want_w = b.dense()
    b.check(out, lse, want_out, want_lse)
    w = b.weights(want_lse.float())
    b.check_weights(w, want_w)


def test_pages_far_beyond_32_bits():
    """A cache of more than 2^32 bytes and 2^31 elements, its live pages at both ends."""
    page, Hk, D = 64, 8, 128
    n_pages = (1 << 31) // (page * Hk * D) + 40
    b = Batch(12, [3], [500], 16, Hk, D, page, BF, spare=0)
    far = [torch.empty(n_pages, page, Hk, D, dtype=BF, device="cuda") for _ in range(2)]
    move = np.where(np.arange(b.n_pages) % 2 == 0, n_pages - 1 - np.arange(b.n_pages), np.arange(b.n_pages))
    for src, dst in ((b.k, far[0]), (b.v, far[1])):
        dst[torch.from_numpy(move).cuda()] = src
    want = b.attend()
    want_w = b.weights(want[1])
    b.table = i32(move[b.table_h])
    b.cache = binding.PagedCache(*far, b.table)
    got = b.attend()
    assert torch.equal(want[0], got[0]) and torch.equal(want[1], got[1]) and torch.equal(want_w, b.weights(want[1]))
    # append and move at the far end
    new = torch.randn(3, Hk, D, device="cuda").to(BF)
    f = torch.zeros(1, dtype=torch.float64, device="cuda")
    binding.rope_append(None, new, new, i32([0, 1, 2]), f, b.cache, b.ctx, b.cu, 3, None)
    for t in range(3):
        s = 500 + t
        p = int(b.table[0, s // page])
        assert torch.equal(far[0][p, s % page], new[t]) and torch.equal(far[1][p, s % page], new[t])
    kept = torch.arange(500, 503, dtype=torch.int32, device="cuda").repeat(1, Hk, 1)
    ko, vo = torch.zeros(1, page, Hk, D, dtype=BF, device="cuda"), torch.zeros(1, page, Hk, D, dtype=BF, device="cuda")
    binding.cache_gather(b.cache, kept, i32([3]), binding.PagedCache(ko, vo, i32([[0]])))
    assert torch.equal(ko[0, :3], new) and torch.equal(vo[0, :3], new)
    assert binding.last_device_status() == 0


def test_pages_that_do_not_exist_are_never_addresses():
    b = Batch(13, [4], [100], 8, 2, 128, 16, BF)
    for bad in (-1, b.n_pages, 2 ** 31 - 1, -2 ** 31):
        table = b.table.clone()
        table[0, 2] = bad
        keep, b.cache = b.cache, binding.PagedCache(b.k, b.v, table)
        assert binding.last_device_status() == 0
        b.attend()
        assert binding.last_device_status() & binding.DEV_PAGE_RANGE
        b.weights(torch.zeros(4, 8, device="cuda"))
        assert binding.last_device_status() & binding.DEV_PAGE_RANGE
        table[0, 6] = bad
        k0 = b.k.clone()
        binding.rope_append(None, b.q[:, :2].contiguous(), b.q[:, :2].contiguous(), i32([0] * 4), torch.zeros(1, dtype=torch.float64, device="cuda"),
                            b.cache, b.ctx, b.cu, 4, None)
        assert binding.last_device_status() & binding.DEV_PAGE_RANGE
        assert torch.equal(torch.nan_to_num(b.k), torch.nan_to_num(k0))
        b.cache = keep
    # a table with too few columns
    keep, b.cache = b.cache, binding.PagedCache(b.k, b.v, b.table[:, :3])
    b.attend()
    assert binding.last_device_status() & binding.DEV_PAGE_RANGE
    b.cache = keep
    out, lse = b.attend()
    b.check(out, lse, *b.dense()[:2])
    assert binding.last_device_status() == 0


def test_lengths_that_do_not_fit_are_recorded():
    b = Batch(14, [4, 3], [100, 20], 8, 2, 128, 16, BF)
    good = b.attend()
    out = torch.zeros_like(good[0])
    b.mt = 3                                       # the first sequence has four tokens: it is left out
    b.attend(out=out)
    assert binding.last_device_status() & binding.DEV_SEQ_RANGE
    assert torch.equal(out[4:], good[0][4:])
    b.mt = 4
    for bad in ([-1, 20], [100, -5], [2 ** 31 - 1, 20], [100, 2 ** 31 - 2], [(1 << 30) + 1, 20]):
        b.ctx = i32(bad)
        b.attend()
        assert binding.last_device_status() & binding.DEV_SEQ_RANGE
        rows = b.q[:, :2].contiguous()
        binding.rope_append(None, rows, rows, i32([0] * b.M), torch.zeros(1, dtype=torch.float64, device="cuda"),
                            binding.PagedCache(b.k.clone(), b.v.clone(), b.table), b.ctx, b.cu, 4, None)
        assert binding.last_device_status() & binding.DEV_SEQ_RANGE
        b.weights(good[1])
        assert binding.last_device_status() & binding.DEV_SEQ_RANGE
    b.ctx = i32([100, 20])
    for cu in ([0, 5, 4], [0, 4, 9], [-1, 4, 7]):
        b.cu = i32(cu)
        b.attend()
        assert binding.last_device_status() & binding.DEV_SEQ_RANGE
    b.cu = i32(b.cu_h)
    b.ml = 90                                       # cut
    b.attend()
    assert binding.last_device_status() & binding.DEV_SEQ_RANGE


@pytest.mark.parametrize("tokens,ctx,Hq,Hk", [([2], [300], 8, 2), ([200], [300], 16, 2), ([1] * 80, [20] * 80, 8, 4)])
def test_waits_that_run_out_are_reported(tokens, ctx, Hq, Hk):
    """The kernels' loads are withheld by the library's diagnostic switch: the first wait for data gives up, the condition is
    reported and cleared, and the next call is correct (nothing is in flight when a kernel gives up)."""
    b = Batch(17, tokens, ctx, Hq, Hk, 128, 16, BF)
    want_out, want_lse, want_w = b.dense()
    assert binding.last_device_status() == 0
    for call in (lambda: b.attend(), lambda: b.weights(want_lse.float())):
        try:
            binding.debug_set_wait(2_000_000, withhold_loads=True)
            call()
            with pytest.raises(binding.AttsError) as err:
                binding.last_device_status()
            assert err.value.status == 9
        finally:
            binding.debug_set_wait(0, withhold_loads=False)
        assert binding.last_device_status() == 0
        b.check(*b.attend(), want_out, want_lse)
        b.check_weights(b.weights(want_lse.float()), want_w)
        assert binding.last_device_status() == 0


@pytest.mark.parametrize("sinks", [0.0, 1.0])
def test_keys_that_stand_out(sinks):
    """A few cached slots far above the rest, late in the cache: the running maximum jumps once, sums before it vanish."""
    b = Batch(18, [5, 60], [700, 1500], 8, 2, 128, 32, FP)
    for s, c in enumerate(b.ctx_h):
        slot = int(c) - 3
        b.k[b.table_h[s, slot // 32], slot % 32] = b.q[int(b.cu_h[s]), ::4] * 2.0 * sinks + 1.0
    out, lse = b.attend()
    want_out, want_lse, want_w = b.dense()
    b.check(out, lse, want_out, want_lse)
    b.check_weights(b.weights(want_lse.float()), want_w)


def test_weights_of_a_tree_with_more_row_tiles_than_are_listed():
    """One head a group and thousands of drafts: more products than a CTA lists ahead."""
    n = 1024 * 3 + 50
    b = Batch(19, [n], [10], 126, 1, 64, 128, BF, tree="fan")        # a token a row tile
    out, lse = b.attend()
    want = b.weights(lse)
    assert want.sum().item() == pytest.approx(n * 126, rel=1e-4)
    pick = [0, 5, 9, 10, 11, 500, n // 2, n + 9]
    par = b.parent
    for slot in pick:
        seen = torch.zeros(n, dtype=torch.bool)
        each = -(-n // 4)
        i = torch.arange(n)
        seen = torch.ones(n, dtype=torch.bool) if slot < 10 else (i >= slot - 10) & (i // each == (slot - 10) // each)
        k = b.k[b.table_h[0, slot // 128], slot % 128, 0].double()
        s = b.q.double() @ k * b.scale
        w = torch.exp(s - lse.double())[seen.cuda()].sum().item()
        assert want[0, 0, slot].item() == pytest.approx(w, rel=1e-4)


def test_on_another_stream_and_in_a_graph():
    b = Batch(15, [12, 30], [800, 60], 16, 4, 128, 16, BF)
    want_out, want_lse, want_w = b.dense()
    b.attend()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        out, lse = b.attend()
        w = b.weights(lse)
    s.synchronize()
    b.check(out, lse, want_out, want_lse)
    b.check_weights(w, want_w)
    ws = torch.empty(binding.tree_attention_workspace_bytes(b.B, b.M, b.Hq, b.Hk, b.D, b.mt, b.ml), dtype=torch.uint8, device="cuda")
    out, lse, w = torch.zeros_like(out), torch.zeros_like(lse), torch.zeros_like(w)
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        binding.tree_attention(b.q, b.cache, b.ctx, b.cu, b.pre, b.end, b.mt, b.ml, b.scale, out, lse, ws)
        binding.cache_weights(b.q, b.cache, lse, b.ctx, b.cu, b.pre, b.end, b.mt, b.ml, b.scale, None, w)
    for _ in range(2):
        out.zero_(), lse.zero_(), w.zero_()
        graph.replay()
        torch.cuda.synchronize()
        b.check(out, lse, want_out, want_lse)
        b.check_weights(w, want_w)


def test_weights_add_up_and_clear_dead_columns():
    b = Batch(16, [6, 2], [90, 300], 8, 2, 128, 16, BF)
    lse = b.attend()[1]
    once = b.weights(lse)
    start = torch.rand(2, 2, b.ml, device="cuda")
    two = b.weights(lse, win=start)
    live = torch.arange(b.ml, device="cuda")[None] < i32(b.len_h)[:, None]
    assert torch.allclose(two[live[:, None].expand_as(two)], (once + start)[live[:, None].expand_as(two)], rtol=2e-7, atol=0)
    assert (two[~live[:, None].expand_as(two)] == 0).all()
    inplace = start.clone()
    binding.cache_weights(b.q, b.cache, lse, b.ctx, b.cu, b.pre, b.end, b.mt, b.ml, b.scale, inplace, inplace)
    assert torch.equal(inplace, two)
    wide = torch.full((2, 2, b.ml + 7), 5.0, device="cuda")
    binding.cache_weights(b.q, b.cache, lse, b.ctx, b.cu, b.pre, b.end, b.mt, b.ml, b.scale, None, wide)
    assert torch.equal(wide[..., :b.ml], once) and (wide[..., b.ml:] == 5.0).all()
    # every row's weights add up to one
    assert once.sum().item() == pytest.approx(b.M * b.Hq, rel=1e-5)


# ---------------------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("D,pairs", [(128, 64), (128, 32), (64, 8), (128, 0), (96, 20), (256, 128), (40, 13), (8, 4)])
@pytest.mark.parametrize("inter", [False, True])
def test_rope_append_against_the_oracle(dtype, D, pairs, inter):
    """Rotation is one rounding of a sum of two products of |x|: u |y| + 2e-6 (|x| + |y|), and fp16's smallest step."""
    rs = np.random.RandomState(D + pairs)
    tokens, ctx, Hq, Hk, page = [5, 0, 1, 9], [3, 8, 0, 27], 6, 2, 8
    b = Batch(21, tokens, ctx, 2, Hk, D, page, dtype)
    M = b.M
    f, mscale = binding.rope_freqs(2 * pairs, 10000.0, "ramp", 4.0, 64)
    pos = rs.randint(-5, 200000, M).astype(np.int32)
    qkv = torch.randn(M, (Hq + 2 * Hk) * D, device="cuda").to(dtype)
    q, k, v = (t.unflatten(1, (-1, D)) for t in qkv.split([Hq * D, Hk * D, Hk * D], dim=1))
    k0, v0 = b.k.clone(), b.v.clone()
    out = torch.full((M, Hq, D), float("nan"), dtype=dtype, device="cuda")
    binding.rope_append(q, k, v, i32(pos), f.cuda(), b.cache, b.ctx, b.cu, b.mt, out, interleaved=inter, mscale=mscale)
    u = UNIT[dtype]
    written = torch.zeros(b.n_pages, page, dtype=torch.bool, device="cuda")

    def close(got, x, p):
        want = orc.rotate(x.double().cpu().numpy(), p, f.numpy(), mscale, inter)
        tol = u * np.abs(want) + 2e-6 * np.abs(x.double().cpu().numpy()).max() + 2.0 ** -25
        assert (np.abs(got.double().cpu().numpy() - want) <= tol).all()
    for s in range(b.B):
        for t in range(tokens[s]):
            i, slot = int(b.cu_h[s]) + t, ctx[s] + t
            page_id = int(b.table_h[s, slot // page])
            written[page_id, slot % page] = True
            close(out[i], q[i], pos[i])
            close(b.k[page_id, slot % page], k[i], pos[i])
            assert torch.equal(b.v[page_id, slot % page], v[i])
    for now, before in ((b.k, k0), (b.v, v0)):
        assert torch.equal(torch.nan_to_num(now[~written]), torch.nan_to_num(before[~written]))
    # in place, and rows that are not 16-byte aligned give the same bits
    odd = torch.zeros(M * (Hq + 2 * Hk) * D + 1, dtype=dtype, device="cuda")[1:].view(M, -1)
    odd.copy_(qkv)
    q2, k2, v2 = (t.unflatten(1, (-1, D)) for t in odd.split([Hq * D, Hk * D, Hk * D], dim=1))
    kw, vw = b.k.clone(), b.v.clone()
    binding.rope_append(q2, k2, v2, i32(pos), f.cuda(), b.cache, b.ctx, b.cu, b.mt + 3, q2, interleaved=inter, mscale=mscale)
    assert torch.equal(q2, out) and torch.equal(torch.nan_to_num(b.k), torch.nan_to_num(kw)) and torch.equal(torch.nan_to_num(b.v), torch.nan_to_num(vw))
    assert binding.last_device_status() == 0


@pytest.mark.parametrize("tokens,Hq,Hk,D", [([500] * 8, 40, 8, 128), ([33] * 70, 28, 4, 128), ([1], 64, 8, 64), ([2000, 3], 5, 1, 128)])
def test_rope_append_at_size(tokens, Hq, Hk, D):
    b = Batch(22, tokens, [17] * len(tokens), Hk, Hk, D, 16, BF, spare=0)
    M = b.M
    f, _ = binding.rope_freqs(D, 1e6)
    pos = i32(np.random.RandomState(1).randint(0, 100000, M))
    q, k, v = (torch.randn(M, h, D, device="cuda").to(BF) for h in (Hq, Hk, Hk))
    out = torch.full_like(q, float("nan"))
    binding.rope_append(q, k, v, pos, f.cuda(), b.cache, b.ctx, b.cu, b.mt, out)
    a = pos.double()[:, None] * f.cuda()
    c, s = torch.cos(a)[:, None], torch.sin(a)[:, None]

    def want(x):
        x, y = x.double().chunk(2, -1)
        return torch.cat([x * c - y * s, y * c + x * s], -1)
    where = torch.from_numpy(np.concatenate([np.arange(t) for t in tokens]) + 17).cuda()
    page = b.table.long()[torch.from_numpy(np.repeat(np.arange(b.B), tokens)).cuda(), where // 16]
    for got, x in ((out, q), (b.k[page, where % 16], k)):
        w = want(x)
        assert ((got.double() - w).abs() <= UNIT[BF] * w.abs() + 1e-5).all()
    assert torch.equal(b.v[page, where % 16], v)


def test_rope_append_refuses_what_does_not_fit():
    b = Batch(23, [2], [3], 2, 2, 64, 8, BF)
    x = torch.zeros(2, 2, 64, dtype=BF, device="cuda")
    f = torch.zeros(4, dtype=torch.float64, device="cuda")
    ok = dict(q=x, k=x, v=x, positions=i32([0, 1]), freqs=f, cache=b.cache, ctx_lens=b.ctx, cu_tokens=b.cu, max_tokens=2, q_out=x.clone())
    for bad in (dict(k=x.half()), dict(k=x[:, :1]), dict(v=x[:1]), dict(q=x[..., :32]), dict(positions=i32([0])), dict(freqs=f.float()),
                dict(positions=torch.zeros(2, dtype=torch.int64, device="cuda")), dict(ctx_lens=i32([1, 2])), dict(cu_tokens=i32([0])),
                dict(k=x.cpu()), dict(v=x.transpose(1, 2).contiguous().transpose(1, 2)), dict(q_out=x[:, :1])):
        with pytest.raises(ValueError):
            binding.rope_append(**{**ok, **bad})
    with pytest.raises(binding.AttsError) as e:
        binding.rope_append(**{**ok, "freqs": torch.zeros(33, dtype=torch.float64, device="cuda")})
    assert e.value.status == 2
    binding.rope_append(**{**ok, "max_tokens": 1})
    assert binding.last_device_status() & binding.DEV_SEQ_RANGE
    with pytest.raises(ValueError):
        binding.PagedCache(b.k, b.v[:, :, :1], b.table)
    with pytest.raises(ValueError):
        binding.PagedCache(b.k, b.v.half(), b.table)
    with pytest.raises(ValueError):
        binding.PagedCache(b.k, b.v, b.table.long())


# ---------------------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("cols,budget,sinks,recent", [(1, 1, 0, 0), (5, 3, 1, 1), (40, 39, 0, 0), (1000, 1000, 4, 10), (1025, 700, 4, 64),
                                                      (5000, 17, 0, 17), (5000, 1, 0, 0), (70001, 20000, 3, 500), (300, 500, 0, 0),
                                                      (2049, 2048, 2000, 48), (140000, 139999, 0, 1)])
@pytest.mark.parametrize("kind", ["spread", "ties", "special"])
def test_select_against_the_oracle(cols, budget, sinks, recent, kind):
    rs = np.random.RandomState(cols)
    B, H = (3, 2) if cols < 10000 else (1, 2)
    lens = [cols, max(cols // 2, 0), 0][:B]
    w = np.exp(rs.randn(B, H, cols) * 3).astype(np.float32)
    if kind == "ties":
        w = rs.randint(0, 3, w.shape).astype(np.float32)
    elif kind == "special":
        w = rs.choice(np.array([np.nan, np.inf, -np.inf, 0.0, -0.0, 1e-45, -1e-45, 3.4e38, -1.0, 2.0], np.float32), w.shape)
    kept = torch.full((B, H, budget), 77, dtype=torch.int32, device="cuda")
    counts = torch.full((B,), 77, dtype=torch.int32, device="cuda")
    binding.cache_select(torch.from_numpy(w).cuda(), i32(lens), budget, sinks, recent, kept, counts)
    got = kept.cpu().numpy()
    for b in range(B):
        for h in range(H):
            want = orc.select(w[b, h], lens[b], budget, sinks, recent)
            assert got[b, h].tolist() == want + [-1] * (budget - len(want))
    assert counts.tolist() == [min(n, budget) for n in lens]
    assert binding.last_device_status() == 0


def test_select_records_lengths_beyond_the_row():
    kept, counts = torch.zeros(2, 1, 4, dtype=torch.int32, device="cuda"), torch.zeros(2, dtype=torch.int32, device="cuda")
    binding.cache_select(torch.arange(20.0, device="cuda").view(2, 1, 10), i32([11, -3]), 4, 0, 0, kept, counts)
    assert binding.last_device_status() & binding.DEV_SEQ_RANGE
    assert counts.tolist() == [4, 0] and kept[0, 0].tolist() == [6, 7, 8, 9] and kept[1, 0].tolist() == [-1] * 4


@pytest.mark.parametrize("D,page,page_out,dtype", [(128, 16, 16, BF), (64, 8, 32, FP), (40, 32, 8, BF), (256, 128, 64, FP)])
def test_gather_moves_rows_and_weights(D, page, page_out, dtype):
    rs = np.random.RandomState(D)
    b = Batch(31, [1, 1, 1], [99, 40, 0], 3, 3, D, page, dtype)
    budget, lens = 50, b.len_h
    counts = np.minimum(lens, budget)
    kept = np.full((3, 3, budget), -1, np.int32)
    for s in range(3):
        for h in range(3):
            kept[s, h, :counts[s]] = np.sort(rs.permutation(lens[s])[:counts[s]])
    per = -(-budget // page_out)
    out_table = rs.permutation(3 * per).reshape(3, per)
    ko, vo = (torch.full((3 * per, page_out, 3, D), 9.0, dtype=dtype, device="cuda") for _ in range(2))
    w = torch.rand(3, 3, 101, device="cuda")
    wo = torch.full((3, 3, budget), 9.0, device="cuda")
    binding.cache_gather(b.cache, i32(kept), i32(counts), binding.PagedCache(ko, vo, i32(out_table)), w, wo)
    for s in range(3):
        for c in range(per * page_out):
            at = int(out_table[s, c // page_out]), c % page_out
            for h in range(3):
                if c < counts[s]:
                    slot = int(kept[s, h, c])
                    src = int(b.table_h[s, slot // page]), slot % page, h
                    assert torch.equal(ko[at][h], b.k[src]) and torch.equal(vo[at][h], b.v[src]) and wo[s, h, c] == w[s, h, slot]
                else:
                    assert (ko[at][h] == 9.0).all() and (vo[at][h] == 9.0).all()
                    assert c >= budget or wo[s, h, c] == 0
    assert binding.last_device_status() == 0
    # slots that are not there are skipped and recorded
    bad = i32(kept)
    bad[0, 0, 0], bad[1, 1, 1], bad[2, 2, 0] = -1, 5000, 2 ** 31 - 1
    binding.cache_gather(b.cache, bad, i32(counts), binding.PagedCache(ko, vo, i32(out_table)), w, wo)
    assert binding.last_device_status() & binding.DEV_PAGE_RANGE
    assert wo[0, 0, 0] == 0 and wo[1, 1, 1] == 0


def test_evicted_cache_attends_like_the_kept_slots():
    """Weights, selection, move and attention in a row: attention over the kept slots alone."""
    b = Batch(32, [4, 7], [400, 350], 8, 2, 128, 16, BF)
    lse = b.attend()[1]
    w = b.weights(lse)
    budget = 100
    kept, counts = torch.empty(2, 2, budget, dtype=torch.int32, device="cuda"), torch.empty(2, dtype=torch.int32, device="cuda")
    binding.cache_select(w, i32(b.ctx_h), budget, 4, 16, kept, counts)
    per = -(-(budget + 8) // 16)
    ko, vo = (torch.full((2 * per, 16, 2, 128), float("nan"), dtype=BF, device="cuda") for _ in range(2))
    small = binding.PagedCache(ko, vo, i32(np.arange(2 * per).reshape(2, per)))
    binding.cache_gather(b.cache, kept, counts, small)
    new = torch.randn(b.M, 2, 128, device="cuda").to(BF)
    binding.rope_append(None, new, new, i32([0] * b.M), torch.zeros(1, dtype=torch.float64, device="cuda"), small, counts, b.cu, b.mt, None)
    c = Batch(33, [4, 7], [budget, budget], 8, 2, 128, 16, BF)
    c.q, c.parent, c.pre, c.end = b.q, b.parent, b.pre, b.end
    c.k, c.v, c.table, c.cache = ko, vo, small.block_table, small
    out, lse = c.attend()
    c.check(out, lse, *c.dense()[:2])
    for s in range(2):                                                  # and the kept slots are the originals
        for h in range(2):
            i = kept[s, h].long()
            want = b.k[b.table[s].long()[i // 16], i % 16, h]
            got = ko[small.block_table[s].long()[torch.arange(budget, device="cuda") // 16], torch.arange(budget, device="cuda") % 16, h]
            assert torch.equal(got, want)


@pytest.mark.parametrize("tree", ["chain", "fan"])
def test_more_drafted_tiles_than_are_listed(tree):
    """Over 131,072 drafted tokens: tiles behind the listed ones are all looked at."""
    n, ctx = 131072 + 900, 5
    b = Batch(20, [n], [ctx], 1, 1, 64, 128, BF, tree=tree)
    out, lse = b.attend()
    k, v = (x[b.table[0].long(), :, 0].flatten(0, 1)[:n + ctx].double() for x in (b.k, b.v))
    each = -(-n // 4) if tree == "fan" else n
    for t in (0, 77, each - 1, n // 2, n - 1):
        first = t // each * each
        seen = torch.cat([torch.arange(ctx), torch.arange(ctx + first, ctx + t + 1)]).cuda()
        s = (b.q[t, 0].double() @ k[seen].T) * b.scale
        want_lse = torch.logsumexp(s, 0)
        want = torch.softmax(s, 0) @ v[seen]
        b.check(out[t:t + 1], lse[t:t + 1], want.view(1, 1, -1), want_lse.view(1, 1))


def test_verification_step_example():
    """examples/verify_step.py end to end against the fp64 definitions of its parts."""
    import importlib.util
    import os
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "verify_step.py")
    spec = importlib.util.spec_from_file_location("verify_step", path)
    ex = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(ex)
    from oracle import atts_oracle

    torch.manual_seed(3)
    target = ex.Target(hidden=256, heads=4, kv_heads=2, head_dim=64, vocab=1000, seed=3)
    samples, slots = 3, 96
    cache = target.new_cache(samples, slots)
    lens = i32([20, 0, 7])
    for b in range(samples):
        for s in range(int(lens[b])):
            p = int(cache.block_table[b, s // 16])
            cache.k[p, s % 16], cache.v[p, s % 16] = (torch.randn(2, 64, device="cuda").to(BF) for _ in range(2))
    parent, cu = [-1, 0, 1, 1, 0, 4, -1, 0, -1, -1], [0, 6, 8, 10]
    x = torch.randn(10, 256, device="cuda").bfloat16()
    ids = torch.randint(0, 1000, (10,), dtype=torch.int32, device="cuda")
    calib = torch.sort(torch.rand(64, device="cuda") + 6.5)[0]
    weights = torch.zeros(samples, 2, slots, device="cuda")
    at = torch.tensor([33, 0, 7])
    r = ex.verify_step(target, cache, lens, at, x, parent, ids, cu, calib, 64, 0.25, weights)
    assert binding.last_device_status() == 0
    assert r["positions"].tolist() == [33, 34, 35, 35, 34, 35, 0, 1, 7, 7]
    # the projection as the library product leaves it, then everything in fp64
    qkv = (x @ target.w_qkv.T).double().cpu().numpy()
    q, f = qkv[:, :256].reshape(10, 4, 64), target.freqs.cpu().numpy()
    rot = np.stack([orc.rotate(q[i], int(r["positions"][i]), f) for i in range(10)])
    host_k, host_v = (c.double().cpu().numpy() for c in (cache.k, cache.v))
    out, lse = orc.tree_attention(rot, host_k, host_v, cache.block_table.cpu().numpy(), [20, 0, 7], cu, np.array(parent), target.scale)
    hidden = x.double().cpu().numpy() + out.reshape(10, -1) @ target.w_out.double().cpu().numpy().T
    # bf16 roundings on the way: rotated queries, probabilities, attention, its projection and the sum, each 2^-8 of its size
    got = r["hidden"].double().cpu().numpy()
    assert np.abs(got - hidden).max() <= 2.0 ** -8 * (4 * np.abs(out).max() * 2 + np.abs(hidden).max())
    lm = target.lm_head.view(torch.int16).cpu().numpy().view(np.uint16)
    want_lp = atts_oracle.token_logprob(r["hidden"].view(torch.int16).cpu().numpy().view(np.uint16), lm, ids.cpu().numpy())
    assert np.abs(r["logprob"].double().cpu().numpy() - want_lp).max() <= 2e-3
    # each of a row's weights add up to one over what it sees: 10 tokens, 4 heads
    assert weights.sum().item() == pytest.approx(40, rel=1e-3)
    smaller, counts, left = ex.evict(target, cache, i32([26, 2, 9]), weights, 12, 2, 3, 32)
    assert counts.tolist() == [12, 2, 9] and left.shape == weights.shape
    assert left[0].sum() <= weights[0].sum() and torch.equal(left[1, :, :2], weights[1, :, :2])
    ex.main()
