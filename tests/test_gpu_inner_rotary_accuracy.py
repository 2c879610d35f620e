"""Sine and cosine of a rotary position, each to its own size, also where it is near 0.

Tolerance: the angle's rest within an eighth of a turn is rounded to fp32 (2^-24 relative), sine and cosine are good to 2 ulp (2^-22): 2^-21
relative.  The reference's angle, position x frequency in fp64, is good to 2^-52 x 10^5 = 2.3e-11."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("rot", [2, 64])
@pytest.mark.parametrize("first", [0, 90000, -100000])
@pytest.mark.parametrize("inverse", [False, True])
def test_sine_and_cosine_to_their_own_size(rot, first, inverse):
    from paper_2508_15706_b200.inner import Rotary
    n = 10000
    q = torch.zeros(1, n, 1, rot, device="cuda")
    q[..., :rot // 2] = 1.0  # (1, 0) of every pair becomes (cos, sin)
    out = torch.empty_like(q)
    Rotary(rot).apply(q, first=first, out_q=out, inverse=inverse)
    pos = torch.arange(n, device="cuda", dtype=torch.float64) + first
    freq = torch.tensor([10000.0 ** (-2.0 * i / rot) for i in range(rot // 2)], dtype=torch.float64, device="cuda")
    angle = pos[:, None] * freq * (-1.0 if inverse else 1.0)
    for got, want in ((out[0, :, 0, :rot // 2], torch.cos(angle)), (out[0, :, 0, rot // 2:], torch.sin(angle))):
        bad = (got.double() - want).abs() > 2.0 ** -21 * want.abs() + 2.4e-11
        assert not torch.any(bad), ((got.double() - want)[bad][:4], want[bad][:4])


def test_quarters_of_a_turn():
    """Whole positions near multiples of a quarter turn: 11 is near 7 of them, 355 near 226."""
    from paper_2508_15706_b200.inner import Rotary
    q = torch.tensor([1.0, 0.0], device="cuda").view(1, 1, 1, 2)
    out = torch.empty_like(q)
    for p in (0, 11, 22, 33, 44, 355, 710, 103993, -355):
        Rotary(2).apply(q, first=p, out_q=out)
        c, s = out.view(2).tolist()
        assert abs(c - math.cos(p)) <= 2.0 ** -21 * abs(math.cos(p)) + 2.4e-11 and abs(s - math.sin(p)) <= 2.0 ** -21 * abs(math.sin(p)) + 2.4e-11
