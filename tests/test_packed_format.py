"""How far what a packed cache holds may be from what was appended: half a scale for channels of at most 14,336 where the group's largest
magnitude is at least 7 * 2^-14, and 2^-15 in smaller groups.

The largest magnitude over 7 is rounded to fp16 (2^-11 of itself) and to three fraction bits (1 / 16 of the scale at most): it is at most
7 * (1 + 1/16) * (1 + 2^-11) = 7.441 scales, so code 7 is its nearest and no channel is off by more than half a scale.  Below 2^-14 scales are
whole multiples of 2^-17 and fp16 numbers of 2^-24: max / 7 is off by (1/2 + 2^-8) 2^-17 at most, the largest channel, cut to 7 scales, by
7 times that, 3.53 * 2^-17, and the others by that or by half a scale of 2^-14 at most: all by no more than 2^-15."""
import numpy as np
import pytest
import torch

from oracle import window_packed_oracle as orc

LEAST, MOST = 7 * 2.0 ** -14, 14336.0


def magnitudes(dtype):
    """Every finite magnitude of the type from its smallest on."""
    x = torch.arange(1, 1 << 15, dtype=torch.int32).to(torch.int16).view(dtype).double().numpy()
    return x[np.isfinite(x)]


def held(group):
    byte, c = orc.quantise(group)
    return orc.scale_of(byte), np.abs(group - c * orc.scale_of(byte))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_groups_from_a_least_magnitude_on_are_held_to_half_a_scale(dtype):
    rs, top = np.random.RandomState(1), magnitudes(dtype)
    top = top[(top >= LEAST) & (top <= MOST)]
    assert top[0] == LEAST and top[-1] == MOST
    for t in np.concatenate([top[:300], top[300:-300:5], top[-300:]]):
        g = torch.from_numpy((2 * rs.rand(32) - 1) * t).to(dtype).double().numpy()
        g[rs.randint(32)] = t
        s, off = held(g)
        assert s >= 2.0 ** -14 and off.max() <= 0.5 * s


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_smaller_groups_are_held_to_a_step_and_not_to_half_a_scale(dtype):
    rs, top = np.random.RandomState(2), magnitudes(dtype)
    worst = 0.0
    for t in top[top < LEAST][::3]:
        g = torch.from_numpy((2 * rs.rand(32) - 1) * t).to(dtype).double().numpy()
        g[rs.randint(32)] = t
        s, off = held(g)
        assert off.max() <= 2.0 ** -15
        worst = max(worst, off.max() / s if s > 0 else 0.0)
    assert worst > 2                                  # (7.5e-5 is held as 5.3e-5: scale 2^-17, cut to 7)
    g = np.zeros(32)
    g[4] = float(torch.tensor(7.5e-5).to(dtype))
    s, off = held(g)
    assert s == 2.0 ** -17 and 2.2e-5 > off[4] > 2.0e-5


def test_magnitudes_beyond_the_largest_are_cut_and_leave_the_others_at_half_a_scale():
    rs = np.random.RandomState(3)
    for t in (14337.0, 30000.0, 65504.0, 3e38):
        g = (2 * rs.rand(32) - 1) * MOST
        g[7] = t
        s, off = held(g)
        assert s == 2048.0 and off[7] == t - MOST and np.delete(off, 7).max() <= 1024
