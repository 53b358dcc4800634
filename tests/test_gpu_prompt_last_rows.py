"""An infinity in the last query's d_out where the sequence ends inside a tile: it reaches that column of dv for every key that the query
sees, as an infinity of its sign (the weights are positive), whatever stands in for the tile's rows behind it."""
import math

import pytest

from tests.test_gpu_prompt import _mods, check, reference
from tests.test_gpu_prompt_hidden import made

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("H,Hk", [(4, 2), (128, 64)])          # waves that share rows, and blocks of 128
@pytest.mark.parametrize("n,past", [(1, 0), (33, 0), (129, 0), (200, 0), (256, 0), (257, 0), (300, 50), (20, 300)])
def test_an_infinity_in_the_last_row(n, past, H, Hk, d, dtype):
    torch, P = _mods()
    dt, q, k, v, do, at = made(torch, n, past, d, dtype, H, Hk)
    out, lse, rest = P.prompt_attention(q, k, v, rest=True, **at)
    want = reference(torch, q, k, v, do, d ** -0.5)
    head = H - 1
    do[n - 1, head, 11], do[n - 1, head, 60] = math.inf, -math.inf
    _, dk, dv = P.prompt_attention_backward(do, q, k, v, out, lse, rest=rest, **at)
    assert bool((dv[:, Hk - 1, 11] == math.inf).all()) and bool((dv[:, Hk - 1, 60] == -math.inf).all())
    hit = torch.zeros_like(dv, dtype=torch.bool)
    hit[:, Hk - 1, 11] = hit[:, Hk - 1, 60] = True
    got = dict(dv=torch.where(hit, want["dv"].to(dt), dv))
    check(torch, got, want, dt, d)
    assert bool(torch.isfinite(dk[:, :Hk - 1]).all()) and bool((~torch.isfinite(dk[:, Hk - 1])).all())
