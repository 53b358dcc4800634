"""The prompt kernels on both sides of the rules that let waves share rows (64 to 256 blocks of 128 rows and heads): the other files'
shapes are nearly all below them, these are above them, at them, or above one and below the other.  Tolerances as in test_gpu_prompt.py."""
import math

import pytest

from tests.test_gpu_prompt import _mods, check, draw, reference, run_packed
from tests.test_gpu_prompt_hidden import BAD, made

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("H,Hk", [(64, 32), (64, 8), (32, 32)])
def test_many_heads(H, Hk, d, dtype):
    torch, P = _mods()
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    nq, nk = [1, 127, 0, 130, 33, 300], [1, 127, 9, 200, 20, 300]
    for n, (got, want) in enumerate(run_packed(torch, P, nq, nk, H, Hk, d, dt)):
        check(torch, got, want, dt, d, what=f"sequence {n}")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("heads", [15, 16, 17, 63, 64, 65])      # of 4 blocks each: 60, 64, 68, 252, 256, 260
def test_both_sides_give_the_same_values(heads, dtype):
    torch, P = _mods()
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    q, k, v, do = (draw(torch, (1, heads, 500, 64), dt, s) for s in (1, 2, 3, 4))
    out, lse, rest = P.prompt_attention(q, k, v, rest=True)
    dq, dk, dv = P.prompt_attention_backward(do, q, k, v, out, lse, rest=rest)
    scores = P.prompt_scores(q, k, lse)
    want = reference(torch, *(x[0].transpose(0, 1) for x in (q, k, v, do)), 64 ** -0.5)
    got = dict(out=out[0].transpose(0, 1), lse=lse[0], scores=scores[0], dq=dq[0].transpose(0, 1), dk=dk[0].transpose(0, 1), dv=dv[0].transpose(0, 1))
    check(torch, got, want, dt, 64)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("H,Hk", [(8, 8), (9, 3), (16, 16), (18, 9)])      # of 16 blocks each: 128 and 288 of queries, 48 to 256 of keys
def test_long_sequences(H, Hk, dtype):
    torch, P = _mods()
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    q, do = draw(torch, (1, H, 2048, 64), dt, 1), draw(torch, (1, H, 2048, 64), dt, 4)
    k, v = draw(torch, (1, Hk, 2048, 64), dt, 2), draw(torch, (1, Hk, 2048, 64), dt, 3)
    out, lse, rest = P.prompt_attention(q, k, v, rest=True)
    dq, dk, dv = P.prompt_attention_backward(do, q, k, v, out, lse, rest=rest)
    scores = P.prompt_scores(q, k, lse)
    want = reference(torch, *(x[0].transpose(0, 1) for x in (q, k, v, do)), 64 ** -0.5)
    got = dict(out=out[0].transpose(0, 1), lse=lse[0], scores=scores[0], dq=dq[0].transpose(0, 1), dk=dk[0].transpose(0, 1), dv=dv[0].transpose(0, 1))
    check(torch, got, want, dt, 64)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("nq,nk", [(1, 3000), (7, 2049), (64, 64), (65, 1000), (33, 97), (1, 1)])
def test_few_queries_behind_many_keys(nq, nk, dtype):
    torch, P = _mods()
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    for d in (64, 128):
        for got, want in run_packed(torch, P, [nq], [nk], 6, 2, d, dt, spare=0):
            check(torch, got, want, dt, d, what=f"d {d}")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("bad", list(BAD))
@pytest.mark.parametrize("n,past,first", [(200, 0, 77), (300, 0, 128), (257, 64, 200)])
def test_hidden_rows_of_many_heads(n, past, first, bad, d, dtype):
    torch, P = _mods()
    dt, q, k, v, do, at = made(torch, n, past, d, dtype, 128, 64)
    late = [x.clone() for x in (q, k, v, do)]
    for x, row in zip(late, (first, first + past, first + past, first)):
        x[row:] = BAD[bad]
    out, lse, rest = P.prompt_attention(*late[:3], rest=True, **at)
    dq, _, _ = P.prompt_attention_backward(late[3], *late[:3], out, lse, rest=rest, **at)
    want = reference(torch, q[:first], k[:first + past], v[:first + past], do[:first], d ** -0.5)
    check(torch, dict(out=out[:first], lse=lse[:, :first], dq=dq[:first]), want, dt, d, what="later rows")
    q[:first], do[:first] = BAD[bad], BAD[bad]
    out, lse, rest = P.prompt_attention(q, k, v, rest=True, **at)
    _, dk, dv = P.prompt_attention_backward(do, q, k, v, out, lse, rest=rest, **at)
    scores = P.prompt_scores(q, k, lse, **at)
    want = reference(torch, q[first:], k, v, do[first:], d ** -0.5)
    keys = slice(first + past, None)
    late = {x: y[:, keys] if x == "scores" else y[keys] if x[:2] in ("dk", "dv") else y for x, y in want.items()}
    check(torch, dict(dk=dk[keys], dv=dv[keys], scores=scores[:, keys]), late, dt, d, what="earlier queries")
    if bad == "nan":
        assert math.isnan(float(dk[:first + past].sum())) and bool(torch.isnan(scores[:, :first + past]).all())
