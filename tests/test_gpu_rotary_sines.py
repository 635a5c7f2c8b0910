"""The angle of a turn is not cut to 32 bits before its sine is taken."""
import math

import pytest
import torch

import block_ref as ref

pytestmark = pytest.mark.gpu

dsv = pytest.importorskip("paper_2502_07590_amd")

DEV = "cuda:0"


@pytest.mark.parametrize("back", [False, True])
@pytest.mark.parametrize("pairs", [64, 37])
def test_what_32_bits_of_an_angle_leave_is_not_lost(pairs, back):
    """The point (1, 0) turned by t: its error along the circle against what rounding t, in turns, to 32 bits leaves of the angle.  Were that lost, the error would
    be minus it and whatever else: a slope of -1.  Where it is turned in afterwards, sine and cosine stand on the grid of 32 bits already and the sum is rounded to it
    again, so that what stays below half a step is lost: a slope of -0.033, formed here by that arithmetic from sines of 64 bits.  The rest, roundings of
    the sines, has nothing to do with it: over n angles the slope is off by 1 / sqrt n of the sizes' ratio, 3 at most (1 to 4 half steps of 2^-24
    against 2^-26 turns / sqrt 3), n above 10^5: 0.02 is twice that."""
    T, d = 4096, 2 * pairs
    g = torch.Generator().manual_seed(1)
    pos = torch.randint(-100000, 100000, (T, 1), generator=g).int()
    freq = ref.freqs([pairs])
    X = torch.zeros(T, 1, d)
    X[..., :pairs] = 1
    p = dsv.Rotary(T, 1, d, "f32", pairs, layout="halves")
    turn = dsv.rotary_bwd if back else dsv.rotary_fwd
    Y = turn(p, X.to(DEV), pos.to(DEV), freq.to(DEV)).cpu().double()[:, 0]
    t = pos.double() * freq
    c, s = torch.cos(t), torch.sin(t)
    turns = t / (2 * math.pi)
    turns -= turns.round()
    near = turns.float().double()
    left = 2 * math.pi * (turns - near)
    assert left.numel() > 1e5 and float(left.square().mean().sqrt()) > 1e-8

    def slope(cos, sin):
        return float((((sin - s) * c - (cos - c) * s) * left).sum() / left.square().sum())

    c0, s0 = (f(2 * math.pi * near).float().double() for f in (torch.cos, torch.sin))
    expected = slope((c0 - s0 * left).float().double(), (s0 + c0 * left).float().double())
    got = slope(Y[:, :pairs], Y[:, pairs:] * (-1 if back else 1))
    assert -0.05 < expected < 0 and abs(got - expected) < 0.02, (got, expected)
