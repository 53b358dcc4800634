"""More queries than keys: the first queries see nothing, may hold anything, and cost next to nothing in the backward pass, wherever in a
tile the first that does see a key lies.  Values and tolerances as in test_gpu_prompt.py."""
import pytest

from tests.test_gpu_prompt import _mods, check, draw, reference
from tests.test_gpu_prompt_hidden import BAD, made

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("H,Hk", [(4, 2), (128, 64)])          # waves that share rows, and blocks of 128
@pytest.mark.parametrize("bad", list(BAD))
@pytest.mark.parametrize("n,without", [(33, 1), (90, 20), (257, 31), (300, 33), (300, 299), (160, 96)])
def test_queries_that_see_nothing(n, without, bad, H, Hk, dtype):
    torch, P = _mods()
    d = 64
    dt, q, k, v, do, at = made(torch, n, -without, d, dtype, H, Hk)
    q[:without], do[:without] = BAD[bad], BAD[bad]
    out, lse, rest = P.prompt_attention(q, k, v, rest=True, **at)
    dq, dk, dv = P.prompt_attention_backward(do, q, k, v, out, lse, rest=rest, **at)
    scores = P.prompt_scores(q, k, lse, **at)
    assert bool((out[:without] == 0).all()) and bool((lse[:, :without] == -float("inf")).all())
    want = reference(torch, q[without:], k, v, do[without:], d ** -0.5)
    check(torch, dict(out=out[without:], lse=lse[:, without:], scores=scores, dq=dq[without:], dk=dk, dv=dv), want, dt, d)


def test_they_cost_next_to_nothing():
    """2048 queries of 32 heads over 8 behind 1900 keys take what 1920 keys do (the first query that sees one lies inside a tile, or at its
    beginning), not a multiple of it."""
    torch, P = _mods()
    times = []
    for keys in (1920, 1900):
        q, do = draw(torch, (4, 32, 2048, 128), torch.bfloat16, 1), draw(torch, (4, 32, 2048, 128), torch.bfloat16, 2)
        k, v = draw(torch, (4, 8, keys, 128), torch.bfloat16, 3), draw(torch, (4, 8, keys, 128), torch.bfloat16, 4)
        out, lse, rest = P.prompt_attention(q, k, v, rest=True)
        best = float("inf")
        for _ in range(5):
            a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
            a.record()
            P.prompt_attention_backward(do, q, k, v, out, lse, rest=rest)
            b.record()
            b.synchronize()
            best = min(best, a.elapsed_time(b))
        times.append(best)
    assert times[1] < 2 * times[0], times
