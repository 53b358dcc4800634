"""Keys that are not finite and that queries do see: a key whose product is minus infinity has weight 0, so that the outputs, the
log-sum-exps, the scores and every gradient are those of the problem without it, but for its own column of dq, where the definition
multiplies that 0 with an infinity.  Values and tolerances as in test_gpu_prompt.py."""
import math

import pytest

from tests.test_gpu_prompt import _mods, check, reference
from tests.test_gpu_prompt_hidden import made

pytestmark = pytest.mark.gpu

# queries, keys in front of them, the key: on the diagonal of a tile of either side, in the tiles before it, in the prefix
SHAPES = [(8, 1, 3), (64, 0, 1), (100, 0, 31), (200, 0, 77), (300, 0, 5), (300, 0, 255), (90, 40, 20), (257, 64, 200)]


def without(torch, q, k, v, do, row, past, scale):
    """reference() of every query's own problem: those from row - past on see the key and do without it, those before see nothing of it."""
    n = len(q)
    first = min(max(row - past, 0), n)
    early = reference(torch, q[:first], k[:first + past], v[:first + past], do[:first], scale) if first else None
    rest = [i for i in range(len(k)) if i != row]
    late = reference(torch, q[first:], k[rest], v[rest], do[first:], scale)
    return first, rest, early, late


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("H,Hk", [(4, 2), (128, 64)])          # waves that share rows, and blocks of 128
@pytest.mark.parametrize("n,past,row", SHAPES)
def test_a_key_of_weight_zero(n, past, row, H, Hk, d, dtype):
    torch, P = _mods()
    dt, q, k, v, do, at = made(torch, n, past, d, dtype, H, Hk)
    at_element = 37
    q[..., at_element] = q[..., at_element].abs() + 0.25       # so that every product with the key is minus infinity
    k[row, :, at_element] = -math.inf
    out, lse, rest = P.prompt_attention(q, k, v, rest=True, **at)
    dq, dk, dv = P.prompt_attention_backward(do, q, k, v, out, lse, rest=rest, **at)
    scores = P.prompt_scores(q, k, lse, **at)
    first, others, early, late = without(torch, q, k, v, do, row, past, d ** -0.5)
    hit = torch.zeros_like(dq, dtype=torch.bool)
    hit[first:, :, at_element] = True
    assert torch.equal(torch.isnan(dq), hit)
    dq = torch.where(hit, torch.zeros_like(dq), dq)
    for part, want in ((slice(0, first), early), (slice(first, n), late)):
        if want is not None:
            for name in ("dq", "dq_g", "dq_p", "dq_o"):
                want[name] = torch.where(hit[part], torch.zeros_like(want[name]), want[name])
            check(torch, dict(out=out[part], lse=lse[:, part], dq=dq[part]), want, dt, d, what=f"queries {part}")
    assert bool((scores[:, row] == 0).all()) and bool((dk[row] == 0).all()) and bool((dv[row] == 0).all())
    if first == 0:                                             # every query sees it: the keys' side is the smaller problem's
        check(torch, dict(dk=dk[others], dv=dv[others], scores=scores[:, others]), late, dt, d, what="keys")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("row", [0, 40, 63, 150])
def test_a_key_that_is_not_a_number(row, dtype):
    """NaN reaches all of what sees the key and nothing before it."""
    torch, P = _mods()
    n, d = 160, 64
    dt, q, k, v, do, at = made(torch, n, 0, d, dtype)
    k[row, 1, 7] = math.nan
    out, lse, rest = P.prompt_attention(q, k, v, rest=True, **at)
    dq, _, _ = P.prompt_attention_backward(do, q, k, v, out, lse, rest=rest, **at)
    hit = torch.zeros((n, 4), dtype=torch.bool, device=q.device)
    hit[row:, 2:] = True
    for x in (out, dq):
        assert torch.equal(torch.isnan(x), hit[..., None].expand_as(x))
    assert torch.equal(torch.isnan(lse), hit.t())
    want = reference(torch, q[:, :2], k[:, :1], v[:, :1], do[:, :2], d ** -0.5)      # the other key head's queries
    check(torch, dict(out=out[:, :2], lse=lse[:2], dq=dq[:, :2]), want, dt, d)
