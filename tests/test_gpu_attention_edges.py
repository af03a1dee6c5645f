"""Attention side at the places where roles of a kernel meet, lengths are cut or a launch takes another form.

Tolerances.  With u the type's unit roundoff, rounding p and then o moves an output by at most u (sum p |v| + |o|); the fp32 part
(scores of magnitude up to 40 off by 2e-5, exponentials and sums by 1e-5) by 1e-4 sum p |v|; fp16 probabilities, carried 2^6
larger and at least 1 at a row's maximum, lose at most 2^-31 each below the type's normal range, n 2^-31 max |v| over n slots.
The roundings are independent and each is spread over at most +-u of its value, u / sqrt(3) in the mean square: so the outputs of
a whole batch are off by at most sqrt((u^2 / 3) (sum p^2 v^2 + o^2)) plus the fp32 part in the mean square, of which 1.2 times is
allowed.  lse and weights: as in test_gpu_attention.py."""
import numpy as np
import pytest
import torch

from oracle import attention_oracle as orc
from paper_2509_15148_b200 import binding
from tests.test_gpu_attention import BF, FP, LARGE, UNIT, Batch, i32

pytestmark = pytest.mark.gpu


class Exact:
    """The definition in fp64 over slots below `cut` (of every sequence): out, lse, weights, sum p |v|, sum p^2 v^2."""

    def __init__(self, b, cut=1 << 30):
        G, f64 = b.Hq // b.Hk, torch.float64
        self.out, self.pv, self.p2v2 = (torch.zeros(b.M, b.Hq, b.D, dtype=f64, device="cuda") for _ in range(3))
        self.lse = torch.full((b.M, b.Hq), -float("inf"), dtype=f64, device="cuda")
        self.w = torch.zeros(b.B, b.Hk, min(b.ml, cut), dtype=f64, device="cuda")
        self.slots, self.vmax = int(b.len_h.max()), torch.nan_to_num(b.v.float()).abs().max().item()
        for s in range(b.B):
            n, c, S = int(b.tokens[s]), int(b.ctx_h[s]), min(int(b.len_h[s]), cut)
            par = b.parent[b.cu_h[s]:b.cu_h[s + 1]]
            see = np.zeros((n, c + n), bool)
            for t in range(n):
                if par[t] != -2:
                    see[t, :c] = True
                    if par[t] >= 0:
                        see[t, c:] = see[par[t], c:]
                    see[t, c + t] = True
            see = torch.from_numpy(see[:, :S]).cuda()
            held = see.any(0)      # what nobody sees may hold anything
            pages = b.table[s, :-(-S // b.page)].long()
            rows = slice(int(b.cu_h[s]), int(b.cu_h[s + 1]))
            for h in range(b.Hk if n else 0):
                heads = slice(h * G, (h + 1) * G)
                k, v = (torch.where(held[:, None], x[pages, :, h].flatten(0, 1)[:S].double(), 0.0) for x in (b.k, b.v))
                x = torch.einsum("tgd,sd->tgs", b.q[rows, heads].double(), k) * b.scale
                x.masked_fill_(~see[:, None], -float("inf"))
                l = torch.logsumexp(x, -1)
                p = torch.exp(x - torch.where(torch.isinf(l), 0.0, l)[..., None])
                self.out[rows, heads], self.lse[rows, heads] = p @ v, l
                self.pv[rows, heads], self.p2v2[rows, heads] = p @ v.abs(), (p * p) @ (v * v)
                self.w[s, h, :S] = p.sum((0, 1))

    def check(self, b, out, lse, rows=slice(None)):
        u, got = UNIT[b.dtype], out[rows].double()
        want, pv, p2v2 = self.out[rows], self.pv[rows], self.p2v2[rows]
        fp32 = 1e-4 * pv + (self.slots * 2.0 ** -31 * self.vmax if b.dtype is FP else 0.0)
        err = (got - want).abs()
        assert not torch.isnan(got).any()
        assert (err <= u * (pv + want.abs()) + fp32).all(), (err - u * (pv + want.abs()) - fp32).max().item()
        rms = lambda x: x.square().mean().sqrt().item()  # noqa: E731
        assert rms(err) <= 1.2 * (rms((u * u / 3 * (p2v2 + want.square())).sqrt()) + rms(fp32)), rms(err)
        dead, want_lse, got_lse = torch.isinf(self.lse[rows]), self.lse[rows], lse[rows].double()
        assert torch.equal(got_lse == -float("inf"), dead)
        assert ((got_lse - want_lse)[~dead].abs() <= 5e-5 + 1e-5 * want_lse[~dead].abs()).all()

    def check_weights(self, b, got):
        e = (got[..., :self.w.shape[-1]].double() - self.w).abs() - 1e-4 * self.w.abs() - 1e-9
        assert not torch.isnan(got).any() and e.max().item() <= 0, e.max().item()


def padded_chains(b, pad):
    """Turns a batch's sequences into chains with padding tokens at the given places, whose slots hold NaN."""
    par = []
    for s, n in enumerate(b.tokens):
        p, last = np.full(n, -2), -1
        for i in range(n):
            if i in pad:
                slot = int(b.ctx_h[s]) + i
                for c in (b.k, b.v):
                    c[b.table_h[s, slot // b.page], slot % b.page] = float("nan")
            else:
                p[i], last = last, i
        par.append(p)
    b.parent = np.concatenate(par).astype(np.int32)
    b.pre, b.end = (x.cuda() for x in binding.tree_plan(b.parent, b.cu_h)[:2])


# One row tile (G = 1, drafts over two slot tiles), many of those (one stream, two CTAs an SM), two row tiles with drafts over two,
# three and four slot tiles.  Every one of those holds padding and the last ends inside, so that they are cleared one after the
# other, behind nothing or behind several cached tiles.
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("tokens,Hq,Hk", [([100], 4, 4), ([120] * 60, 4, 4), ([200], 8, 2), ([330], 8, 2), ([460], 8, 2), ([460, 17, 300], 5, 1)])
@pytest.mark.parametrize("ctx", [0, 60, 1000])
def test_several_tiles_with_padding_in_a_row(D, tokens, Hq, Hk, ctx):
    b = Batch(41, tokens, [ctx] * len(tokens), Hq, Hk, D, 16, BF)
    padded_chains(b, set(range(5, 460, 40)))
    want = Exact(b)
    assert binding.last_device_status() == 0
    for _ in range(3):
        out, lse = b.attend()
        assert binding.last_device_status() == 0
        want.check(b, out, lse)
    want.check_weights(b, b.weights(want.lse.float()))


@pytest.mark.parametrize("count", [-3, -300, -2 ** 31, 601, 2 ** 31 - 1])
def test_gather_cuts_and_records_counts_that_do_not_fit(count):
    """kept_cols = 600: blocks that begin beyond the count, and beyond their first one."""
    b = Batch(42, [1, 1], [700, 650], 2, 2, 64, 16, BF)
    kept = torch.arange(600, dtype=torch.int32, device="cuda").repeat(2, 2, 1)
    ko, vo = (torch.full((80, 16, 2, 64), 9.0, dtype=BF, device="cuda") for _ in range(2))
    dst = binding.PagedCache(ko, vo, torch.arange(80, dtype=torch.int32, device="cuda").view(2, 40))
    w, wo = torch.rand(2, 2, 700, device="cuda"), torch.full((2, 2, 600), 9.0, device="cuda")
    assert binding.last_device_status() == 0
    binding.cache_gather(b.cache, kept, torch.tensor([count, 5], dtype=torch.int32, device="cuda"), dst, w, wo)
    assert binding.last_device_status() == binding.DEV_SEQ_RANGE
    n = 600 if count > 0 else 0
    slot = torch.arange(600, device="cuda")
    pages = b.table.long()[:, slot // 16]
    for got, src in ((ko, b.k), (vo, b.v)):
        first, second = got.view(2, 640, 2, 64)
        assert torch.equal(first[:n], src[pages[0], slot % 16][:n]) and (first[n:] == 9.0).all()
        assert torch.equal(second[:5], src[pages[1], slot % 16][:5]) and (second[5:] == 9.0).all()
    assert torch.equal(wo[0, :, :n], w[0, :, :n]) and (wo[0, :, n:] == 0).all()
    assert torch.equal(wo[1, :, :5], w[1, :, :5]) and (wo[1, :, 5:] == 0).all()


@pytest.mark.parametrize("tree", ["chain", "random"])
@pytest.mark.parametrize("tokens,ctx,cut,Hq,Hk,D", [([2], [300], 200, 8, 2, 128), ([200], [300], 200, 8, 2, 64), ([4, 9], [5000, 40], 4999, 8, 2, 128),
                                                    ([4], [300], 256, 8, 2, 128), ([3] * 200, [250] * 200, 130, 8, 4, 128), ([150], [1000], 1100, 8, 2, 64)])
def test_sequences_cut_at_max_len_see_exactly_the_slots_below_it(tokens, ctx, cut, Hq, Hk, D, tree):
    b = Batch(43, tokens, ctx, Hq, Hk, D, 16, BF, tree=tree)
    want = Exact(b, cut)
    b.ml = cut
    out, lse = b.attend()
    assert binding.last_device_status() == binding.DEV_SEQ_RANGE
    want.check(b, out, lse)
    want.check_weights(b, b.weights(want.lse.float()))
    assert binding.last_device_status() == binding.DEV_SEQ_RANGE


# one row tile, and more than one
@pytest.mark.parametrize("tokens,ctx,Hq,Hk", [([4, 3], [100, 300], 8, 2), ([150, 90], [300, 260], 8, 2)])
@pytest.mark.parametrize("bad", ["ctx", "tokens", "cu"])
def test_weights_of_a_sequence_that_does_not_fit_stay(tokens, ctx, Hq, Hk, bad):
    b = Batch(44, tokens, ctx, Hq, Hk, 128, 16, BF)
    want = Exact(b)
    lse = want.lse.float()
    if bad == "ctx":
        b.ctx = i32([-1, ctx[1]])
    elif bad == "tokens":
        b.mt = tokens[0] - 1
    else:
        b.cu = i32([-1] + b.cu_h[1:].tolist())
    before = torch.rand(2, Hk, b.ml, device="cuda")
    for inplace in (False, True):
        win = before.clone()
        out = win if inplace else torch.full_like(win, float("nan"))
        binding.cache_weights(b.q, b.cache, lse, b.ctx, b.cu, b.pre, b.end, b.mt, b.ml, b.scale, win, out)
        assert binding.last_device_status() == binding.DEV_SEQ_RANGE
        assert torch.equal(out[0], before[0])
        n = int(b.len_h[1])
        assert ((out[1, :, :n].double() - before[1, :, :n].double() - want.w[1, :, :n]).abs() <= 1e-4 * want.w[1, :, :n] + 1e-6).all()
        assert (out[1, :, n:] == 0).all()
    out = torch.full_like(before, float("nan"))
    binding.cache_weights(b.q, b.cache, lse, b.ctx, b.cu, b.pre, b.end, b.mt, b.ml, b.scale, None, out)
    assert binding.last_device_status() == binding.DEV_SEQ_RANGE and (out[0] == 0).all()


# one chunk and several, one row tile, two, and many sequences
@pytest.mark.parametrize("tokens,ctx,Hq,Hk", [([5], [40], 8, 2), ([5], [9000], 8, 2), ([200], [300], 8, 2), ([3] * 90, [200] * 90, 8, 2)])
@pytest.mark.parametrize("D,dtype", [(128, BF), (64, FP)])
@pytest.mark.parametrize("where", ["query", "key", "score"])
def test_nan_and_infinity_reach_the_rows_that_see_them(tokens, ctx, Hq, Hk, D, dtype, where):
    """A row is hit where one of its scores is NaN or +inf (a NaN channel of its query, a NaN key, a product that overflows); every
    other row stays exact."""
    b = Batch(45, tokens, ctx, Hq, Hk, D, 16, dtype, tree="chain")
    hit = torch.zeros(b.M, Hq, dtype=torch.bool, device="cuda")
    want = Exact(b)
    if where == "key":       # the first sequence's third token: it and its descendants, the heads of key head 1
        slot = int(b.ctx_h[0]) + 2
        b.k[b.table_h[0, slot // 16], slot % 16, 1, 3] = float("nan")
        hit[2:tokens[0], Hq // Hk:] = True
    else:                    # the first sequence's second token, query head 3
        hit[1, 3] = True
        if where == "query":
            b.q[1, 3, 7] = float("nan")
        else:                # (a key channel of exactly 1 or -1 in every slot: the score is inf or -inf, some of them inf)
            b.q[1, 3] = 0
            b.q[1, 3, 0] = float("inf")
            assert (b.k[b.table_h[0, 0], :, 0, 0] > 0).any()
    out, lse = b.attend()
    assert binding.last_device_status() == 0
    assert torch.equal(torch.isnan(lse), hit) and torch.equal(torch.isnan(out), hit[..., None].expand_as(out))
    keep = (~hit).all(1)
    want.check(b, out, lse, keep)


@pytest.mark.parametrize("case", LARGE + [
    # few rows over long caches in both types and head sizes: chunks joined
    ([4], [30000], 8, 2, 64, 32, BF, "random", 0.0),
    ([4], [30000], 8, 2, 64, 32, FP, "random", 0.0),
    ([13, 9], [70000, 41000], 8, 2, 128, 64, BF, "random", 0.0),
    ([13, 9], [70000, 41000], 8, 2, 128, 64, FP, "random", 0.0),
    ([150], [50000], 4, 2, 128, 128, BF, "fan", 0.0)])
def test_outputs_at_size_within_their_own_bound(case):
    """Over tens of thousands of slots outputs are small: the allowance goes by sum p |v| and, in the mean square, by sum p^2 v^2."""
    tokens, ctx, Hq, Hk, D, page, dtype, tree, pad = case
    b = Batch(46, tokens, ctx, Hq, Hk, D, page, dtype, tree, pad)
    want = Exact(b)
    out, lse = b.attend()
    assert binding.last_device_status() == 0
    want.check(b, out, lse)
    want.check_weights(b, b.weights(want.lse.float()))


@pytest.mark.parametrize("tree", ["chain", "fan"])
def test_tiles_behind_the_listed_ones(tree):
    """131,972 drafts of two heads: one chunk of 1032 slot tiles, 1024 of which are listed; the last eight are looked at by all."""
    n, ctx = 131072 + 900, 5
    assert binding.tree_attention_workspace_bytes(1, n, 2, 2, 64, n, n + ctx) == 256       # one chunk
    b = Batch(47, [n], [ctx], 2, 2, 64, 128, BF, tree=tree)
    out, lse = b.attend()
    assert binding.last_device_status() == 0
    each = -(-n // 4) if tree == "fan" else n
    for h in range(2):
        k, v = (x[b.table[0].long(), :, h].flatten(0, 1)[:n + ctx].double() for x in (b.k, b.v))
        for t in (0, 1000, each - 1, n // 2, n - 1000, n - 900, n - 700, n - 1):
            first = t // each * each
            seen = torch.cat([torch.arange(ctx), torch.arange(ctx + first, ctx + t + 1)]).cuda()
            s = (b.q[t, h].double() @ k[seen].T) * b.scale
            p = torch.softmax(s, 0)
            want, pv = p @ v[seen], p @ v[seen].abs()
            assert ((out[t, h].double() - want).abs() <= UNIT[BF] * (pv + want.abs()) + 1e-4 * pv).all()
            assert abs(lse[t, h].item() - torch.logsumexp(s, 0).item()) <= 5e-5 + 1e-5 * abs(lse[t, h].item())


@pytest.mark.parametrize("tokens", [[1201, 999, 0, 1, 2600], [7000], [160] * 31])
@pytest.mark.parametrize("D,pairs,inter", [(128, 64, False), (128, 32, True), (64, 8, False), (96, 20, True), (128, 0, False)])
@pytest.mark.parametrize("dtype", [BF, FP])
def test_rope_append_of_many_tokens(tokens, D, pairs, inter, dtype):
    """From 4736 tokens on (148 SMs) a block takes four of them; lengths that are not multiples of four.  One rounding of a sum of two
    products of |x|: u |y| + 2e-6 max |x| + fp16's smallest step, cosine and sine in fp64 here."""
    Hq, Hk, page = 6, 2, 16
    ctx = [(37 * i) % 100 for i in range(len(tokens))]
    b = Batch(48, tokens, ctx, Hk, Hk, D, page, dtype, tree="chain")
    assert b.M >= 4736
    f = binding.rope_freqs(2 * pairs, 10000.0)[0].cuda()
    pos = torch.randint(-5, 200000, (b.M,), dtype=torch.int32, device="cuda")
    qkv = torch.randn(b.M, (Hq + 2 * Hk) * D, device="cuda").to(dtype)
    q, k, v = (t.unflatten(1, (-1, D)) for t in qkv.split([Hq * D, Hk * D, Hk * D], dim=1))
    k0, v0 = b.k.clone(), b.v.clone()
    angle = pos.double()[:, None] * f
    c, s = torch.cos(angle)[:, None], torch.sin(angle)[:, None]

    def want(x):
        x = x.double()
        y = x.clone()
        one, two = (slice(0, 2 * pairs, 2), slice(1, 2 * pairs, 2)) if inter else (slice(0, pairs), slice(pairs, 2 * pairs))
        y[..., one], y[..., two] = x[..., one] * c - x[..., two] * s, x[..., two] * c + x[..., one] * s
        return y
    seq = torch.from_numpy(np.repeat(np.arange(b.B), tokens)).cuda()
    slot = torch.from_numpy(np.concatenate([np.arange(t) + x for t, x in zip(tokens, ctx)])).cuda()
    pages = b.table.long()[seq, slot // page]
    touched = torch.zeros(b.n_pages, page, dtype=torch.bool, device="cuda")
    touched[pages, slot % page] = True
    odd = torch.zeros(qkv.numel() + 1, dtype=dtype, device="cuda")[1:].view_as(qkv)
    odd.copy_(qkv)
    for rows in (qkv, odd):          # aligned, and not
        qq, kk, vv = (t.unflatten(1, (-1, D)) for t in rows.split([Hq * D, Hk * D, Hk * D], dim=1))
        out = torch.full((b.M, Hq, D), float("nan"), dtype=dtype, device="cuda")
        b.k.copy_(k0), b.v.copy_(v0)
        binding.rope_append(qq, kk, vv, pos, f, b.cache, b.ctx, b.cu, b.mt, out, interleaved=inter)
        assert binding.last_device_status() == 0
        for got, x in ((out, q), (b.k[pages, slot % page], k)):
            w = want(x)
            assert ((got.double() - w).abs() <= UNIT[dtype] * w.abs() + 2e-6 * x.double().abs().max() + 2.0 ** -25).all()
        assert torch.equal(b.v[pages, slot % page], v)
        for now, before in ((b.k, k0), (b.v, v0)):
            assert torch.equal(torch.nan_to_num(now[~touched]), torch.nan_to_num(before[~touched]))


@pytest.mark.parametrize("cols,budget,sinks,recent", [(4097, 4096, 4, 100), (9000, 1, 0, 0), (16384, 8000, 4, 512), (16385, 8192, 4, 512), (20001, 20000, 0, 0),
                                                      (32000, 8192, 4, 512), (32767, 1, 0, 0), (32768, 16384, 0, 16384), (32768, 31000, 7, 0),
                                                      (32769, 8192, 4, 512)])
@pytest.mark.parametrize("kind", ["spread", "ties", "special", "equal"])
def test_select_on_rows_of_every_form(cols, budget, sinks, recent, kind):
    """Clusters of two with 8 and 16 keys a thread, their first and last row lengths, and the first of the long form."""
    rs = np.random.RandomState(cols + budget)
    lens = [cols, cols - 1, max(budget, cols // 2), budget + 1, 0]
    B, H = len(lens), 2
    w = np.exp(rs.randn(B, H, cols) * 3).astype(np.float32)
    if kind == "ties":
        w = rs.randint(0, 3, w.shape).astype(np.float32)
    elif kind == "special":
        w = rs.choice(np.array([np.nan, np.inf, -np.inf, 0.0, -0.0, 1e-45, -1e-45, 3.4e38, -1.0, 2.0], np.float32), w.shape)
    elif kind == "equal":
        w[:] = 0.25
    kept = torch.full((B, H, budget), 77, dtype=torch.int32, device="cuda")
    counts = torch.full((B,), 77, dtype=torch.int32, device="cuda")
    binding.cache_select(torch.from_numpy(w).cuda(), i32(lens), budget, sinks, recent, kept, counts)
    got = kept.cpu().numpy()
    for s in range(B):
        for h in range(H):
            want = orc.select(w[s, h], lens[s], budget, sinks, recent)
            assert got[s, h].tolist() == want + [-1] * (budget - len(want))
    assert counts.tolist() == [min(n, budget) for n in lens]
    assert binding.last_device_status() == 0


def test_batches_without_tokens_or_sequences():
    """No drafts at all: attention and append do nothing, weights are carried over.  No sequences: nothing is done."""
    b = Batch(49, [2, 1], [100, 30], 8, 2, 128, 16, BF)
    none, cu = torch.empty(0, 8, 128, dtype=BF, device="cuda"), i32([0, 0, 0])
    e = i32(np.zeros(0))
    kv = torch.empty(0, 2, 128, dtype=BF, device="cuda")
    f = torch.zeros(4, dtype=torch.float64, device="cuda")
    ws = torch.empty(binding.tree_attention_workspace_bytes(2, 0, 8, 2, 128, 0, 103), dtype=torch.uint8, device="cuda")
    lse = torch.empty(0, 8, device="cuda")
    k0 = b.k.clone()
    binding.rope_append(none, kv, kv, e, f, b.cache, b.ctx, cu, 0, none)
    binding.tree_attention(none, b.cache, b.ctx, cu, e, e, 0, 103, 0.1, none, lse, ws)
    win = torch.rand(2, 2, 110, device="cuda")
    for bounds in (0, 5):
        out = torch.full_like(win, 7.0)
        binding.cache_weights(none, b.cache, lse, b.ctx, cu, None, None, bounds, 103, 0.1, win, out)
        for s, n in enumerate((100, 30)):
            assert torch.equal(out[s, :, :n], win[s, :, :n]) and (out[s, :, n:103] == 0).all() and (out[s, :, 103:] == 7).all()
    assert torch.equal(torch.nan_to_num(b.k), torch.nan_to_num(k0))
    empty = binding.PagedCache(b.k, b.v, torch.empty(0, 4, dtype=torch.int32, device="cuda"))
    zero = i32([0])
    binding.rope_append(none, kv, kv, e, f, empty, e, zero, 0, none)
    binding.tree_attention(none, empty, e, zero, None, None, 0, 0, 0.1, none, lse, ws)
    w = torch.empty(0, 2, 10, device="cuda")
    binding.cache_weights(none, empty, lse, e, zero, None, None, 0, 10, 0.1, None, w)
    kept = torch.empty(0, 2, 5, dtype=torch.int32, device="cuda")
    binding.cache_select(w, e, 5, 0, 0, kept, e)
    binding.cache_gather(empty, kept, e, empty)
    assert binding.last_device_status() == 0
