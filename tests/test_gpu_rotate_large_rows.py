"""Norms of rows whose squares add up to more than fp32 holds though their mean does not (the mean and eps together are a normal number), the
formula and tolerances of test_gpu_rotate.py: scaling by a power of two costs no rounding."""
import pytest

from tests.test_gpu_rotate import DEV, Formula, _mods, both_ways, draw, dtype_of

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
def test_squares_beyond_fp32(d, dtype):
    torch, P = _mods()
    dt = dtype_of(torch, dtype)
    q, k = draw(torch, (40, 4, d), dt, 1), draw(torch, (40, 2, d), dt, 2)
    q[1], k[2] = q[1] * 6e18, k[2] * 6e18                        # squares of 4e37 each, some of them beyond 2^128
    q[3, 1], q[3, 1, 7] = 0.0, 1e20                              # one element whose square is
    q[4, 2, 5] = 1e19                                            # only the sum of 1e38 and what is smaller by far
    k[5] = 1.2e19 * torch.sign(k[5].float()).to(dt)              # a mean of 1.4e38
    pos = torch.arange(40, dtype=torch.int32, device=DEV)
    w = 1.0 + 0.3 * draw(torch, (d,), torch.float32, 3)
    f, rotary = Formula(torch, pos, d, d), P.Rotary(d)
    both_ways(torch, P, q, k, pos, f, rotary, dt, qw=w, kw=w + 0.5)
    both_ways(torch, P, q, k[:, :1] * 0.01, pos, f, rotary, dt, qw=w)
