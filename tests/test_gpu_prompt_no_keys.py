"""Gradients of queries that see nothing: an empty sum, zero whatever their rows and those of d_out hold."""
import pytest

from tests.test_gpu_prompt import _mods
from tests.test_gpu_prompt_hidden import BAD, made

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("H,Hk", [(4, 2), (128, 64)])          # waves that share rows, and blocks of 128
@pytest.mark.parametrize("bad", list(BAD))
@pytest.mark.parametrize("n,without", [(1, 1), (33, 1), (90, 20), (257, 31), (300, 299), (160, 96)])
def test_gradients_of_queries_that_see_nothing(n, without, bad, H, Hk, d, dtype):
    torch, P = _mods()
    dt, q, k, v, do, at = made(torch, n, -without, d, dtype, H, Hk)
    clean = P.prompt_attention_backward(do, q, k, v, *P.prompt_attention(q, k, v, **at), **at)[0]
    q[:without], do[:without] = BAD[bad], BAD[bad]
    out, lse, rest = P.prompt_attention(q, k, v, rest=True, **at)
    dq, _, _ = P.prompt_attention_backward(do, q, k, v, out, lse, **at)
    assert bool((clean[:without] == 0).all()) and bool((dq[:without] == 0).all())
    assert bool(torch.isfinite(dq[without:]).all())
