"""Long rows of the cache in 4 bits, so many that finishing threads have two and four slots each (other files' rows leave them one)."""
import pytest

from tests.test_gpu_q4 import _mods, compare, made, take_step

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("H,Hk,K", [(60, 60, 4100), (120, 60, 4100), (130, 130, 4097)])      # 5 x 60 > 256, 3 x 130 > 256
def test_steps(H, Hk, K):
    torch, P = _mods()
    dt = torch.bfloat16
    cache, m = made(torch, P, 1, H, Hk, 64, K, 40, dt, [K + 300])
    for i in range(2):
        take_step(torch, cache, m, dt, 100 + 10 * i, f"step {i}")
    compare(torch, cache, m, "after")
