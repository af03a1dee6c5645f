"""Host side of the attention operators: numbering of draft trees, rotary frequencies, refusals of arguments, and pins of
the fp64 oracle."""
import ctypes
import math

import numpy as np
import pytest
import torch

from oracle import attention_oracle as orc
from paper_2509_15148_b200 import binding


def random_parents(rs, T, pad=0.0):
    par = np.array([-1] + [rs.randint(-1, i) for i in range(1, T)], np.int32)[:T]
    dead = rs.rand(T) < pad
    par[dead] = -2
    for i in range(T):
        if par[i] >= 0 and par[par[i]] == -2:
            par[i] = -1
    return par


@pytest.mark.parametrize("T", [0, 1, 2, 3, 17, 130])
@pytest.mark.parametrize("pad", [0.0, 0.3])
def test_tree_plan_intervals_are_ancestry(T, pad):
    rs = np.random.RandomState(T)
    par = np.concatenate([random_parents(rs, T, pad), random_parents(rs, T, pad)])
    pre, end, depth = (x.numpy() for x in binding.tree_plan(par, [0, T, 2 * T]))
    for off in (0, T):
        for i in range(T):
            seen = [j for j in range(T) if pre[off + j] <= pre[off + i] < end[off + j]]
            assert seen == orc.visible(par[off:off + T], i)
            assert depth[off + i] == max(len(seen) - 1, 0)
        live = pre[off:off + T][par[off:off + T] != -2]
        assert sorted(live) == list(range(len(live)))


def test_tree_plan_refusals():
    for par in ([0], [-3], [-1, 1], [-1, 2, 0], [-2, 0]):
        with pytest.raises(binding.AttsError) as e:
            binding.tree_plan(par, [0, len(par)])
        assert e.value.status == 6
    with pytest.raises(ValueError):
        binding.tree_plan([-1, 0], [0, 1])
    with pytest.raises(binding.AttsError):
        binding.tree_plan([-1, 0], [0, 3, 2])
    with pytest.raises(binding.AttsError):
        binding.tree_plan([-1], [1, 1])


def test_rope_freqs():
    f, m = binding.rope_freqs(8, 10000.0)
    assert m == 1.0 and np.allclose(f.numpy(), [1.0, 0.1, 0.01, 0.001], rtol=1e-14)
    g, _ = binding.rope_freqs(8, 10000.0, "linear", 4.0)
    assert torch.equal(g, f / 4)
    # bands: turns over 1000 positions are 159, 15.9, 1.59, 0.159; low 1, high 4
    g, m = binding.rope_freqs(8, 10000.0, "bands", 8.0, 1000, 1.0, 4.0)
    keep = (1000 * 0.01 / (2 * math.pi) - 1) / 3
    assert m == 1.0 and np.allclose(g.numpy(), [1.0, 0.1, 0.01 * keep + 0.01 / 8 * (1 - keep), 0.001 / 8], rtol=1e-14)
    # ramp: channel where 1000 positions make n turns is 8 ln(1000 / (2 pi n)) / (2 ln 10000)
    lo = max(math.floor(8 * math.log(1000 / (2 * math.pi * 32)) / (2 * math.log(1e4))), 0)
    hi = math.ceil(8 * math.log(1000 / (2 * math.pi)) / (2 * math.log(1e4)))
    g, m = binding.rope_freqs(8, 10000.0, "ramp", 8.0, 1000)
    ramp = np.clip((np.arange(4) - lo) / (hi - lo), 0, 1)
    assert m == pytest.approx(0.1 * math.log(8) + 1) and np.allclose(g.numpy(), f.numpy() * (1 - ramp + ramp / 8), rtol=1e-14)
    assert binding.rope_freqs(0)[0].numel() == 0
    for bad in (dict(rotary_dim=7), dict(rotary_dim=8, base=0.0), dict(rotary_dim=8, scaling="other"),
                dict(rotary_dim=8, scaling="bands", low=4.0, high=4.0), dict(rotary_dim=8, factor=0.0)):
        with pytest.raises(ValueError):
            binding.rope_freqs(**bad)


def test_oracle_rotation_is_a_rotation():
    rs = np.random.RandomState(3)
    x, y = rs.randn(16), rs.randn(16)
    f = binding.rope_freqs(12, 500.0)[0].numpy()
    for inter in (False, True):
        a, b = orc.rotate(x, 70, f, 1.0, inter), orc.rotate(y, 64, f, 1.0, inter)
        c, d = orc.rotate(x, 6, f, 1.0, inter), orc.rotate(y, 0, f, 1.0, inter)
        assert np.dot(a, b) == pytest.approx(np.dot(c, d), rel=1e-12)        # only the distance matters
        assert np.array_equal(a[12:], x[12:]) and np.array_equal(d, y)
        assert np.allclose(orc.rotate(orc.rotate(x, 9, f, 1.0, inter), -9, f, 1.0, inter), x, rtol=1e-13)


def test_oracle_attention_against_closed_forms():
    rs = np.random.RandomState(4)
    k, v = np.zeros((4, 8, 1, 8)), rs.randn(4, 8, 1, 8)
    table = np.array([[2, 0, 3, 1]])
    q = rs.randn(3, 2, 8)
    par = np.array([-1, -1, -2])
    out, lse = orc.tree_attention(q, k, v, table, [9], [0, 3], par, 0.3)
    rows = [v[2, i, 0] for i in range(8)] + [v[0, 0, 0]]
    assert np.allclose(out[0, 0], np.mean(rows + [v[0, 1, 0]], 0)) and np.allclose(out[1, 1], np.mean(rows + [v[0, 2, 0]], 0))
    assert np.allclose(lse[:2], math.log(10)) and np.all(out[2] == 0) and np.all(np.isneginf(lse[2]))
    w = orc.cache_weights(q, k, table, lse, [9], [0, 3], par, 0.3, 14)
    assert np.allclose(w[0, 0], [0.4] * 9 + [0.2, 0.2, 0, 0, 0])


def test_oracle_selection():
    w = [0.5, 0.0, 2.0, 2.0, float("nan"), 1.0, -0.0, 0.25]
    assert orc.select(w, 8, 3, 0, 0) == [2, 3, 5]
    assert orc.select(w, 8, 2, 0, 1) == [2, 7]
    assert orc.select(w, 8, 4, 2, 1) == [0, 1, 2, 7]
    assert orc.select(w, 8, 7, 0, 0) == [0, 1, 2, 3, 5, 6, 7]
    assert orc.select(w, 2, 3, 0, 0) == [0, 1]


def _cache(**kw):
    c = binding._KvCache(256, 256, 256, 2, 4, 4, 8, 16, 16 * 8 * 128, 8 * 128, 128, 8, 128, 0, 0)
    for n, x in kw.items():
        setattr(c, n, x)
    return ctypes.addressof(c), c


def test_cache_descriptions_are_checked_before_the_device():
    lib = binding.load()

    def gather(**kw):
        ref, keep = _cache(**kw)
        good, keep2 = _cache()
        return lib.atts_cache_gather(ref, None, 0, 256, good, None, 0, None, None)

    for kw, status in ((dict(dtype=2), 6), (dict(reserved=1), 6), (dict(heads=0), 2), (dict(head_dim=12), 2), (dict(head_dim=264), 2),
                       (dict(page_size=24), 2), (dict(page_size=4), 2), (dict(page_size=8192), 2), (dict(num_pages=-1), 2),
                       (dict(table_cols=-1), 2), (dict(table_stride=3), 2), (dict(page_stride=12), 2), (dict(slot_stride=-8), 2),
                       (dict(head_stride=4), 2), (dict(k=None), 1), (dict(v=None), 1), (dict(block_table=None), 1), (dict(k=264), 3),
                       (dict(block_table=258), 3), (dict(num_seqs=65536), 2), (dict(num_seqs=1), 2), (dict(heads=4), 2), (dict(dtype=1), 6)):
        assert gather(**kw) == status, kw
    assert lib.atts_cache_gather(None, None, 0, None, None, None, 0, None, None) == 1


def _attend(lib, cache=None, q=256, q_ts=4096, q_hs=128, ctx=256, cu=256, pre=None, end=None, M=4, Hq=32, mt=4, ml=64, scale=0.1,
            out=256, o_ts=4096, lse=None, ws=256, wsb=1 << 40):
    ref, keep = cache or _cache()
    return lib.atts_tree_attention(q, q_ts, q_hs, ref, ctx, cu, pre, end, M, Hq, mt, ml, scale, out, o_ts, 128, lse, ws, wsb, None)


def test_tree_attention_refusals():
    lib = binding.load()
    for kw, status in ((dict(Hq=12), 2), (dict(Hq=0), 2), (dict(Hq=8 * 129), 2), (dict(M=-1), 2), (dict(mt=-1), 2), (dict(mt=65), 2),
                       (dict(ml=(1 << 30) + 1), 2), (dict(q_ts=4097), 2), (dict(q_hs=-8), 2), (dict(o_ts=4), 2), (dict(scale=0.0), 6),
                       (dict(scale=-1.0), 6), (dict(scale=float("nan")), 6), (dict(scale=float("inf")), 6), (dict(q=None), 1),
                       (dict(out=None), 1), (dict(ctx=None), 1), (dict(cu=None), 1), (dict(pre=256), 1), (dict(end=256), 1),
                       (dict(ws=None), 1), (dict(q=264), 3), (dict(out=260), 3), (dict(ws=128), 3), (dict(lse=2), 3), (dict(ctx=257), 3),
                       (dict(cache=_cache(head_dim=96)), 2), (dict(cache=_cache(head_dim=256)), 2)):
        assert _attend(lib, **kw) == status, kw
    sz = ctypes.c_size_t(0)
    assert lib.atts_tree_attention_workspace_bytes(1, 1, 32, 8, 128, 1, 100, None) == 1
    for bad in ((-1, 1, 32, 8, 128, 1, 9), (1, 1, 30, 8, 128, 1, 9), (1, 1, 32, 8, 80, 1, 9), (1, 1, 32, 8, 128, 10, 9), (1, -1, 32, 8, 128, 1, 9)):
        assert lib.atts_tree_attention_workspace_bytes(*bad, ctypes.byref(sz)) == 2


def test_rope_weights_and_select_refusals():
    lib = binding.load()
    ref, keep = _cache()

    def rope(q=256, k=256, v=256, pos=256, freqs=256, pairs=64, mscale=1.0, inter=0, ctx=256, cu=256, M=4, Hq=32, mt=4, out=256, ks=1024):
        return lib.atts_rope_append(q, 4096, 128, k, ks, 128, v, 1024, 128, pos, freqs, pairs, mscale, inter, ref, ctx, cu, M, Hq, mt,
                                    out, 4096, 128, None)
    for kw, status in ((dict(pairs=65), 2), (dict(pairs=-1), 2), (dict(M=-1), 2), (dict(Hq=-1), 2), (dict(mt=-1), 2), (dict(ks=-8), 2),
                       (dict(inter=2), 6), (dict(mscale=float("nan")), 6), (dict(mscale=float("inf")), 6), (dict(q=None), 1),
                       (dict(out=None), 1), (dict(k=None), 1), (dict(v=None), 1), (dict(pos=None), 1), (dict(freqs=None), 1),
                       (dict(ctx=None), 1), (dict(cu=None), 1), (dict(k=257), 3), (dict(freqs=260), 3), (dict(pos=258), 3)):
        assert rope(**kw) == status, kw

    def weights(lse=256, wout=256, cols=64, ml=64, win=None, Hq=32):
        return lib.atts_cache_weights(256, 4096, 128, ref, lse, 256, 256, None, None, 4, Hq, 4, ml, 0.1, win, wout, cols, None)
    for kw, status in ((dict(lse=None), 1), (dict(wout=None), 1), (dict(cols=63), 2), (dict(lse=258), 3), (dict(wout=258), 3),
                       (dict(win=258), 3), (dict(Hq=33), 2)):
        assert weights(**kw) == status, kw

    def select(w=256, cols=64, lens=256, B=2, heads=8, budget=10, sinks=2, recent=3, kept=256, counts=256):
        return lib.atts_cache_select(w, cols, lens, B, heads, budget, sinks, recent, kept, counts, None)
    for kw, status in ((dict(budget=0), 2), (dict(sinks=-1), 2), (dict(recent=-1), 2), (dict(sinks=8), 2), (dict(cols=-1), 2),
                       (dict(B=-1), 2), (dict(heads=0), 2), (dict(w=None), 1), (dict(lens=None), 1), (dict(kept=None), 1),
                       (dict(counts=None), 1), (dict(w=258), 3), (dict(kept=258), 3)):
        assert select(**kw) == status, kw
