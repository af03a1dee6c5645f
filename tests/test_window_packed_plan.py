"""Pins of the definitions of the normed rotation, the window and the cache in 4 bits, and refusals of their entry points (host only)."""
import ctypes
import math

import numpy as np
import pytest
import torch

from oracle import window_packed_oracle as orc
from paper_2509_15148_b200 import binding
from tests.test_attention_arguments import BF, F32, F64, GPU0, GPU1, HOST, I32, U8, Tensor, calls  # noqa: F401


# ---- definitions ------------------------------------------------------------------------------------------------------
def test_norm_makes_unit_mean_square_and_rotation_keeps_it():
    x = np.random.RandomState(0).randn(5, 64) * 3
    y = orc.norm_rotate(x, np.ones(64), 0.0, 17, [1.0, 0.1, 0.01])
    assert np.allclose((y * y).mean(-1), 1.0)
    assert np.allclose(orc.norm_rotate(x, None, 0.0, 0, [1.0]), x)


def test_window_of_a_chain_is_the_last_places_and_the_sinks():
    see = orc.sees(np.arange(-1, 5), 10, window=4, sinks=2)
    for t in range(6):
        want = [s for s in range(16) if s <= 10 + t and (s > 10 + t - 4 or s < 2)]
        assert np.flatnonzero(see[t]).tolist() == want


def test_window_follows_a_tokens_own_line():
    # tokens 0-1-2 and a second branch 3-4 from the cache: slot 10 + 4 has place 11
    see = orc.sees([-1, 0, 1, -1, 3], 10, window=3, sinks=0)
    assert np.flatnonzero(see[2]).tolist() == [10, 11, 12]
    assert np.flatnonzero(see[4]).tolist() == [9, 13, 14]
    assert np.flatnonzero(orc.sees([-1, -2], 3, window=2)[1]).tolist() == []


def test_a_sink_may_be_a_drafted_token():
    see = orc.sees([-1, 0, 1, 2], 1, window=1, sinks=3)
    assert np.flatnonzero(see[3]).tolist() == [0, 1, 2, 4]


def test_scales_are_the_upper_bits_of_fp16():
    for b in range(209):
        h = np.array([b << 7], np.uint16).view(np.float16)[0]
        assert float(h) == orc.scale_of(b)
    assert orc.scale_of(208) == 2048.0 and math.isnan(orc.scale_of(255)) and np.isnan(np.array([255 << 7], np.uint16).view(np.float16)[0])


def test_quantised_groups_by_hand():
    x = np.zeros(32)
    assert orc.quantise(x)[0] == 0
    x[3] = 7.0                                       # scale 1: ties at halves go to even
    x[:3] = 2.5, 3.5, -0.5
    byte, c = orc.quantise(x)
    assert orc.scale_of(byte) == 1.0 and c[:4].tolist() == [2, 4, 0, 7]
    x[3] = 14336.0 * 4
    byte, c = orc.quantise(x)
    assert orc.scale_of(byte) == 2048.0 and c[3] == 7
    x[5] = math.inf
    assert orc.quantise(x)[0] == 255


def test_what_is_held_is_within_half_a_scale_and_exact_in_sixteen_bits():
    rs = np.random.RandomState(1)
    for mag in (1e-3, 1.0, 300.0):
        x = torch.from_numpy(rs.randn(64, 32) * mag).bfloat16().double().numpy()
        for g in x:
            byte, c = orc.quantise(g)
            s = orc.scale_of(byte)
            assert np.abs(g - c * s).max() <= 0.75 * s        # half a scale, and what a scale below max / 7 cuts off (7 / 16 at most)
            for t in (torch.bfloat16, torch.float16):
                assert torch.equal(torch.from_numpy(c * s).to(t).double(), torch.from_numpy(c * s))


def test_packing_round_trips():
    x = torch.from_numpy(np.random.RandomState(2).randn(16, 64)).half().double().numpy()
    block = np.full(binding.packed_block_bytes(16, 64), 0xAA, np.uint8)
    for e in range(16):
        codes, scales = orc.packed_slot(x[e])
        c0, s0 = orc.slot_bytes(e, 64)
        block[c0:c0 + 32], block[s0:s0 + 2] = codes, scales
    want = np.array([np.concatenate([orc.scale_of(b) * c for b, c in (orc.quantise(r[g:g + 32]) for g in (0, 32))]) for r in x])
    assert np.array_equal(orc.unpack(block, 16, 64), want)


# ---- refusals of the library: before anything touches a device ---------------------------------------------------------
def kv(**over):
    f = dict(k=4096, v=4096, block_table=4096, num_seqs=2, table_cols=4, table_stride=4, num_pages=8, page_size=16, page_stride=16 * 2 * 64,
             slot_stride=2 * 64, head_stride=64, heads=2, head_dim=64, dtype=0, reserved=0)
    return binding._KvCache(**{**f, **over})


def packed(**over):
    block = 16 * (32 + 2)
    f = dict(k=4096, v=4096, block_table=4096, num_seqs=2, table_cols=4, table_stride=4, num_pages=8, page_size=16, page_stride=2 * block,
             head_stride=block, heads=2, head_dim=64)
    return binding._PackedCache(**{**f, **over})


def ref(c):
    return None if c is None else ctypes.addressof(c)


def attention(name, cache, **over):
    a = dict(q=4096, qt=4 * 64, qh=64, dtype=0, ctx=4096, cu=4096, pre=4096, end=4096, depth=4096, window=8, sinks=2, M=6, Hq=4, mt=3, ml=50, scale=0.1,
             out=4096, ot=4 * 64, oh=64, lse=4096, ws=4096, wsb=0)
    a.update(over)
    mid = (a["dtype"],) if name == "packed" else ()
    return getattr(binding.load(), f"atts_{name}_attention")(
        a["q"], a["qt"], a["qh"], *mid, ref(cache), a["ctx"], a["cu"], a["pre"], a["end"], a["depth"], a["window"], a["sinks"], a["M"], a["Hq"], a["mt"],
        a["ml"], a["scale"], a["out"], a["ot"], a["oh"], a["lse"], a["ws"], a["wsb"], None)


NULL, SHAPE, ALIGN, ARG = 1, 2, 3, 6


@pytest.mark.parametrize("name", ["window", "packed"])
@pytest.mark.parametrize("over, status", [
    (dict(window=-1), ARG), (dict(window=(1 << 30) + 1), ARG), (dict(sinks=-1), ARG), (dict(sinks=(1 << 30) + 1), ARG),
    (dict(depth=None), NULL), (dict(pre=None, end=None), NULL), (dict(pre=None), NULL), (dict(depth=4098), ALIGN),
    (dict(Hq=3), SHAPE), (dict(M=-1), SHAPE), (dict(mt=60), SHAPE), (dict(qt=4), SHAPE), (dict(qh=0), SHAPE), (dict(scale=0.0), ARG),
    (dict(scale=float("nan")), ARG), (dict(q=None), NULL), (dict(q=4098), ALIGN), (dict(out=None), NULL), (dict(ws=None), NULL), (dict(ws=4100), ALIGN),
    (dict(ot=12), SHAPE), (dict(lse=4098), ALIGN), (dict(ml=(1 << 30) + 1), SHAPE)])
def test_attention_refuses(name, over, status):
    assert attention(name, kv() if name == "window" else packed(), **over) == status


def test_a_window_of_none_is_for_packed_caches_only():
    assert attention("window", kv(), window=0) == ARG
    assert attention("packed", packed(), window=0, depth=None, dtype=7) == ARG
    assert attention("packed", packed(head_dim=192, head_stride=16 * 102, page_stride=2 * 16 * 102)) == SHAPE     # attention: 64 or 128


PACKED_BAD = [(dict(head_dim=32), SHAPE), (dict(head_dim=96), SHAPE), (dict(head_dim=320), SHAPE), (dict(page_size=12), SHAPE), (dict(page_size=4), SHAPE),
              (dict(page_size=8192), SHAPE), (dict(heads=0), SHAPE), (dict(num_seqs=65536), SHAPE), (dict(page_stride=1096), SHAPE), (dict(head_stride=528), SHAPE),
              (dict(head_stride=-544), SHAPE), (dict(num_pages=1 << 31), SHAPE), (dict(table_stride=3), SHAPE), (dict(k=None), NULL), (dict(block_table=None), NULL),
              (dict(k=4104), ALIGN), (dict(block_table=4098), ALIGN)]


@pytest.mark.parametrize("over, status", PACKED_BAD + [(None, NULL)])
def test_packed_descriptions_are_refused(over, status):
    lib, c = binding.load(), None if over is None else packed(**over)
    assert attention("packed", c) == status
    assert lib.atts_packed_append(4096, 128, 64, 4096, 128, 64, 0, ref(c), 4096, 4096, 6, 3, None) == status
    d = kv()
    assert lib.atts_packed_read(ref(c), 4096, 50, ref(d), None) == status


@pytest.mark.parametrize("over, status", [(dict(dtype=2), ARG), (dict(M=-1), SHAPE), (dict(mt=-1), SHAPE), (dict(kt=-8), SHAPE), (dict(k=None), NULL), (dict(v=None), NULL),
                                          (dict(ctx=None), NULL), (dict(cu=None), NULL), (dict(k=4097), ALIGN), (dict(cu=4098), ALIGN)])
def test_packed_append_refuses(over, status):
    a = dict(k=4096, kt=128, v=4096, dtype=0, ctx=4096, cu=4096, M=6, mt=3)
    a.update(over)
    c = packed()
    assert binding.load().atts_packed_append(a["k"], a["kt"], 64, a["v"], 128, 64, a["dtype"], ref(c), a["ctx"], a["cu"], a["M"], a["mt"], None) == status


@pytest.mark.parametrize("dst, over, status", [(dict(heads=1), {}, SHAPE), (dict(head_dim=128), {}, SHAPE), (dict(num_seqs=3), {}, SHAPE), (dict(dtype=3), {}, ARG),
                                               ({}, dict(ml=-1), SHAPE), ({}, dict(lens=None), NULL), ({}, dict(lens=4098), ALIGN)])
def test_packed_read_refuses(dst, over, status):
    a = dict(lens=4096, ml=50)
    a.update(over)
    c, d = packed(), kv(**dst)
    assert binding.load().atts_packed_read(ref(c), a["lens"], a["ml"], ref(d), None) == status


NORM = dict(q=4096, qt=256, k=4096, kt=128, v=4096, pos=4096, freqs=4096, pairs=32, ms=1.0, inter=0, qg=4096, kg=4096, eps=1e-6, ctx=4096, cu=4096, M=6, Hq=4,
            mt=3, out=4096)


@pytest.mark.parametrize("over, status", [
    (dict(pairs=33), SHAPE), (dict(pairs=-1), SHAPE), (dict(eps=-1.0), ARG), (dict(eps=float("inf")), ARG), (dict(eps=float("nan")), ARG), (dict(ms=float("inf")), ARG),
    (dict(inter=2), ARG), (dict(M=-1), SHAPE), (dict(Hq=-1), SHAPE), (dict(qt=-8), SHAPE), (dict(q=None), NULL), (dict(k=None), NULL), (dict(pos=None), NULL),
    (dict(freqs=None), NULL), (dict(out=None), NULL), (dict(qg=4097), ALIGN), (dict(kg=4097), ALIGN), (dict(pos=4098), ALIGN), (dict(freqs=4100), ALIGN)])
def test_normed_rotations_refuse(over, status):
    a = {**NORM, **over}
    lib, c = binding.load(), kv()
    turned = (a["pos"], a["freqs"], a["pairs"], a["ms"], a["inter"], a["qg"], a["kg"], a["eps"])
    assert lib.atts_norm_rope_append(a["q"], a["qt"], 64, a["k"], a["kt"], 64, a["v"], 128, 64, *turned, ref(c), a["ctx"], a["cu"], a["M"], a["Hq"], a["mt"], a["out"],
                                     256, 64, None) == status
    assert lib.atts_norm_rope(a["q"], a["qt"], 64, a["k"], a["kt"], 64, *turned, 0, a["M"], a["Hq"], 2, 64, a["out"], 256, 64, 4096, 128, 64, None) == status


def test_normed_rotations_refuse_what_is_their_own():
    lib, c = binding.load(), kv()
    a = NORM
    turned = (a["pos"], a["freqs"], a["pairs"], a["ms"], a["inter"], a["qg"], a["kg"], a["eps"])
    append = lambda v, ctx, mt: lib.atts_norm_rope_append(4096, 256, 64, 4096, 128, 64, v, 128, 64, *turned, ref(c), ctx, 4096, 6, 4, mt, 4096, 256, 64, None)  # noqa: E731
    assert append(None, 4096, 3) == NULL and append(4096, None, 3) == NULL and append(4096, 4096, -1) == SHAPE and append(4097, 4096, 3) == ALIGN
    rows = lambda dtype, D, k_out, kt: lib.atts_norm_rope(4096, 256, 64, 4096, 128, 64, *turned, dtype, 6, 4, 2, D, 4096, 256, 64, k_out, kt, 64, None)  # noqa: E731
    assert rows(2, 64, 4096, 128) == ARG and rows(0, 60, 4096, 128) == SHAPE and rows(0, 264, 4096, 128) == SHAPE
    assert rows(0, 64, None, 128) == NULL and rows(0, 64, 4096, -8) == SHAPE and rows(0, 64, 4097, 128) == ALIGN


@pytest.mark.parametrize("name", ["window", "packed"])
def test_workspace_sizes_refuse(name):
    f, n = getattr(binding.load(), f"atts_{name}_attention_workspace_bytes"), ctypes.c_size_t(0)
    good = [2, 6, 4, 2, 64, 3, 50, 8, 2]
    for at, bad, status in ((0, -1, SHAPE), (2, 3, SHAPE), (4, 96, SHAPE), (5, 60, SHAPE), (6, (1 << 30) + 1, SHAPE), (7, -1, ARG), (8, -1, ARG), (7, (1 << 30) + 1, ARG)):
        args = list(good)
        args[at] = bad
        assert f(*args, ctypes.byref(n)) == status
    assert f(*good, None) == NULL


# ---- the binding: tensors of another device, of another type or shape never reach the library -----------------------------
def handles(dev):
    block = binding.packed_block_bytes(16, 64)
    if dev.type != "cuda":
        return None, None
    return (binding.PagedCache(Tensor((4, 16, 2, 64), BF, dev), Tensor((4, 16, 2, 64), BF, dev), Tensor((2, 2), I32, dev)),
            binding.PackedCache(Tensor((4, 2, block), U8, dev), Tensor((4, 2, block), U8, dev), Tensor((2, 2), I32, dev), 16, 64))


def arguments(dev):
    t = lambda *s, d=I32: Tensor(s, d, dev)  # noqa: E731
    q, kv, lens, cu, gain = t(3, 4, 64, d=BF), t(3, 2, 64, d=BF), t(2), t(3), t(64, d=BF)
    c, p = handles(dev)
    attn = dict(q=q, ctx_lens=lens, cu_tokens=cu, pre=t(3), end=t(3), depth=t(3), window=8, sinks=1, max_tokens=2, max_len=32, scale=0.1, out=q,
                lse=t(3, 4, d=F32), workspace=t(4096, d=U8))
    turn = dict(positions=t(3), freqs=t(32, d=F64), q_gain=gain, k_gain=gain, eps=1e-6)
    return {
        "norm_rope_append": (binding.norm_rope_append, dict(q=q, k=kv, v=kv, **turn, cache=c, ctx_lens=lens, cu_tokens=cu, max_tokens=2, q_out=q)),
        "norm_rope": (binding.norm_rope, dict(q=q, k=kv, **turn, q_out=q, k_out=kv)),
        "window_attention": (binding.window_attention, dict(cache=c, **attn)),
        "packed_attention": (binding.packed_attention, dict(cache=p, **attn)),
        "packed_append": (binding.packed_append, dict(k=kv, v=kv, cache=p, ctx_lens=lens, cu_tokens=cu, max_tokens=2)),
        "packed_read": (binding.packed_read, dict(src=p, lens=lens, max_len=32, dst=c)),
    }


NAMES = sorted(arguments(GPU0))


@pytest.mark.parametrize("name", NAMES)
def test_tensors_of_the_current_device_reach_the_library(calls, name):  # noqa: F811
    f, args = arguments(GPU0)[name]
    f(**args)
    assert calls == ["atts_" + name]


@pytest.mark.parametrize("name", NAMES)
def test_tensors_of_another_device_are_refused(calls, name):  # noqa: F811
    f, args = arguments(GPU1)[name]
    with pytest.raises(ValueError):
        f(**args)
    assert calls == []


@pytest.mark.parametrize("name", NAMES)
@pytest.mark.parametrize("other", [GPU1, HOST])
def test_one_tensor_elsewhere_of_another_type_or_size_is_refused(calls, name, other):  # noqa: F811
    f, args = arguments(GPU0)[name]
    for key, x in args.items():
        if isinstance(x, Tensor):
            bad = [Tensor(x.shape, x.dtype, other)]
            if key != "workspace":
                bad += [Tensor((x.shape[0] + 1,) + tuple(x.shape[1:]), x.dtype), Tensor(x.shape, torch.int64)]
            if key == "freqs":
                bad.pop(1)             # any number of pairs has a meaning
            for b in bad:
                with pytest.raises(ValueError):
                    f(**{**args, key: b})
        elif isinstance(x, (binding.PagedCache, binding.PackedCache)) and other.type == "cuda":
            with pytest.raises(ValueError):
                f(**{**args, key: handles(other)[0 if isinstance(x, binding.PagedCache) else 1]})
    assert calls == []


@pytest.mark.parametrize("bad", [dict(k=Tensor((4, 2, 543), U8)), dict(k=Tensor((4, 2, 544), torch.int8)), dict(v=Tensor((4, 1, 544), U8)), dict(page_size=24),
                                 dict(head_dim=96), dict(block_table=Tensor((2, 2), torch.int64)), dict(block_table=Tensor((2,), I32)),
                                 dict(k=Tensor((4, 2, 544), U8, HOST), v=Tensor((4, 2, 544), U8, HOST)), dict(v=Tensor((4, 2, 544), U8, GPU1))])
def test_packed_handles_refuse(bad):
    good = dict(k=Tensor((4, 2, 544), U8), v=Tensor((4, 2, 544), U8), block_table=Tensor((2, 2), I32), page_size=16, head_dim=64)
    binding.PackedCache(**good)
    with pytest.raises(ValueError):
        binding.PackedCache(**{**good, **bad})
