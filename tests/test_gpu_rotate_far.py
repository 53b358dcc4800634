"""Rotation at the largest positions, with angles from frequencies in 80 decimal digits and whole turns dropped exactly (not from the table that the
kernel reads).

Tolerance: 4 f (|a| + |b|) as in test_gpu_rotate.py, and what the angle is off by as include/adore.h states it, 2^-33 + |position| (2^-65 + 2^-62 of the
frequency) turns, times 2 pi."""
import math
from fractions import Fraction

import pytest

from tests.test_gpu_rotate import DEV, F, _mods, draw, near
from tests.test_rotate_turns_cpu import exact_turns

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("R,how", [(64, dict()), (128, dict(base=500000.0)), (128, dict(factor=8.0, original=4096.0)), (48, dict(base=1.0)),
                                   (16, dict(base=0.01)), (64, dict(base=1e-4, factor=0.5))])
def test_angles_at_the_largest_positions(R, how):
    torch, P = _mods()
    pos = [2 ** 31 - 1, -2 ** 31, 2 ** 30 + 12345, -1999999999, 7]
    d = 128 if R > 64 else 64
    x = draw(torch, (len(pos), 2, d), torch.float32, 1)
    got, _ = P.rotate_heads(x, None, torch.tensor(pos, dtype=torch.int32, device=DEV), P.Rotary(R, **how))
    turns = [Fraction(t) for t in exact_turns(R, **how)]
    for i, p in enumerate(pos):
        t = torch.tensor([2 * math.pi * float(p * f % 1) for f in turns], dtype=torch.float64, device=DEV)
        angle = torch.tensor([2 * math.pi * (2.0 ** -33 + abs(p) * (2.0 ** -65 + float(f) * 2.0 ** -62)) for f in turns], dtype=torch.float64, device=DEV)
        a, b = x[i, :, :R].double().split(R // 2, -1)
        want = torch.cat([a * t.cos() - b * t.sin(), a * t.sin() + b * t.cos()], -1)
        off = (4 * F + angle) * (a.abs() + b.abs())
        near(torch, got[i, :, :R], want, torch.cat([off, off], -1), torch.float32, f"position {p}")
        assert torch.equal(got[i, :, R:], x[i, :, R:])
