"""Rows in front of the first sequence: they belong to none, and are zeros (log-sum-exp: minus infinity) like those behind the last one."""
import math

import pytest

from tests.test_gpu_prompt import DEV, _mods, check, draw, reference

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("H,Hk", [(4, 2), (64, 32)])
@pytest.mark.parametrize("front,lengths,behind", [(1, [5], 0), (130, [40, 0, 129], 3), (127, [1], 127), (7, [0, 0], 0), (31, [33, 64, 1, 1], 31),
                                                  (500, [3], 1), (64, [200], 64)])
def test_rows_in_front_of_the_first_sequence(front, lengths, behind, H, Hk, dtype):
    torch, P = _mods()
    dt, d = torch.bfloat16 if dtype == "bf16" else torch.float32, 64
    starts = [front]
    for n in lengths:
        starts.append(starts[-1] + n)
    T = starts[-1] + behind
    q, k, v, do = (draw(torch, (T, h, d), dt, s) for h, s in ((H, 1), (Hk, 2), (Hk, 3), (H, 4)))
    start = torch.tensor(starts, dtype=torch.int32, device=DEV)
    at = dict(q_start=start, k_start=start)
    out, lse, rest = P.prompt_attention(q, k, v, out=torch.full_like(q, 7.0), rest=True, **at)
    dq, dk, dv = P.prompt_attention_backward(do, q, k, v, out, lse, rest=rest, dq=torch.full_like(q, 7.0), dk=torch.full_like(k, 7.0),
                                             dv=torch.full_like(v, 7.0), **at)
    scores = P.prompt_scores(q, k, lse, scores=torch.full((Hk, T), 7.0, device=DEV), **at)
    for none in (slice(0, front), slice(starts[-1], T)):
        for x in (out, dq, dk, dv, scores.t()):
            assert bool((x[none] == 0).all())
        assert bool((lse[:, none] == -math.inf).all())
        assert rest is None or bool((rest[none] == 0).all())
    for a, b in zip(starts, starts[1:]):
        i = slice(a, b)
        want = reference(torch, q[i], k[i], v[i], do[i], d ** -0.5)
        check(torch, dict(out=out[i], lse=lse[:, i], scores=scores[:, i], dq=dq[i], dk=dk[i], dv=dv[i]), want, dt, d)
