"""Scales so small that all weights of a row are equal, down to the least that fp32 holds: rows see their keys all the same.
Tolerances as in test_gpu_prompt.py."""
import pytest

from tests.test_gpu_prompt import _mods, check, run_packed

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("H,Hk", [(4, 2), (128, 64)])          # waves that share rows, and blocks of 128
@pytest.mark.parametrize("scale", [2.0 ** -120, 1.2e-38, 1e-38, 1e-44])
def test_small_scales(scale, H, Hk, dtype):
    torch, P = _mods()
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    for n, (got, want) in enumerate(run_packed(torch, P, [1, 140], [1, 200], H, Hk, 64, dt, scale=scale)):
        check(torch, got, want, dt, 64, what=f"sequence {n}")
