"""Rows that a mask hides may hold anything: infinities and NaN in later keys and values, and in earlier queries, reach nothing that
does not see them, and everything that does.  Values and tolerances as in test_gpu_prompt.py: those of the problem without the rows."""
import math

import pytest

from tests.test_gpu_prompt import DEV, _mods, check, draw, reference

pytestmark = pytest.mark.gpu

# queries, keys in front of them (negative: the first queries see none), first row that is not finite
SHAPES = [(40, 0, 1), (200, 0, 77), (130, 0, 64), (300, 0, 128), (100, 37, 50), (257, 64, 200), (90, -20, 55)]
BAD = {"nan": math.nan, "inf": math.inf, "-inf": -math.inf}


def made(torch, n, past, d, dtype, H=4, Hk=2):
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    q, do = draw(torch, (n, H, d), dt, 1), draw(torch, (n, H, d), dt, 4)
    k, v = draw(torch, (n + past, Hk, d), dt, 2), draw(torch, (n + past, Hk, d), dt, 3)
    at = dict(q_start=torch.tensor([0, n], dtype=torch.int32, device=DEV), k_start=torch.tensor([0, n + past], dtype=torch.int32, device=DEV))
    return dt, q, k, v, do, at


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("bad", list(BAD))
@pytest.mark.parametrize("n,past,first", SHAPES)
def test_later_rows_reach_no_earlier_query(n, past, first, bad, d, dtype):
    """As behind the ends of a batch's shorter sequences, in buffers that nobody has cleared."""
    torch, P = _mods()
    dt, q, k, v, do, at = made(torch, n, past, d, dtype)
    for x, row in ((q, first), (do, first), (k, first + past), (v, first + past)):
        x[row:] = BAD[bad]
    out, lse, rest = P.prompt_attention(q, k, v, rest=True, **at)
    dq, _, _ = P.prompt_attention_backward(do, q, k, v, out, lse, rest=rest, **at)
    want = reference(torch, q[:first], k[:first + past], v[:first + past], do[:first], d ** -0.5)
    check(torch, dict(out=out[:first], lse=lse[:, :first], dq=dq[:first]), want, dt, d, what="out")
    assert bool((~torch.isfinite(out[first:])).all()) and bool((~torch.isfinite(lse[:, first:])).all()) or bad != "nan"


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("bad", list(BAD))
@pytest.mark.parametrize("n,past,first", SHAPES)
def test_earlier_queries_reach_no_later_key(n, past, first, bad, d, dtype):
    torch, P = _mods()
    dt, q, k, v, do, at = made(torch, n, past, d, dtype)
    q[:first], do[:first] = BAD[bad], BAD[bad]
    out, lse, rest = P.prompt_attention(q, k, v, rest=True, **at)
    dq, dk, dv = P.prompt_attention_backward(do, q, k, v, out, lse, rest=rest, **at)
    scores = P.prompt_scores(q, k, lse, **at)
    want = reference(torch, q[first:], k, v, do[first:], d ** -0.5)
    keys = slice(first + past, None)
    got = dict(out=out[first:], lse=lse[:, first:], dq=dq[first:])
    check(torch, got, want, dt, d, what="out")
    got = dict(dk=dk[keys], dv=dv[keys], scores=scores[:, keys])
    late = {x: y[:, keys] if x == "scores" else y[keys] if x[:2] in ("dk", "dv") else y for x, y in want.items()}
    check(torch, got, late, dt, d, what="keys")
    if bad == "nan":                                   # (keys before: every one is seen by such a query)
        seen = slice(0, max(0, first + past))
        assert bool(torch.isnan(dk[seen]).all()) and bool(torch.isnan(dv[seen]).all()) and bool(torch.isnan(scores[:, seen]).all())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("bad", list(BAD))
def test_one_element_reaches_what_sees_it(bad, dtype):
    """One element of V, and of d_out: its column of the rows that see it, nothing else of out and dv."""
    torch, P = _mods()
    n, d, H, Hk = 190, 64, 4, 2
    for row in (0, 1, 63, 64, 100, 188, 189):
        dt, q, k, v, do, at = made(torch, n, 0, d, dtype, H, Hk)
        want = reference(torch, q, k, v, do, d ** -0.5)
        spoilt = v.clone()
        spoilt[row, 1, 37] = BAD[bad]
        out, lse = P.prompt_attention(q, k, spoilt, **at)
        finite = torch.isfinite(out)
        hit = torch.zeros_like(finite)
        hit[row:, 2:, 37] = True
        assert torch.equal(~finite, hit), row
        check(torch, dict(out=torch.where(hit, want["out"].to(dt), out), lse=lse), want, dt, d, what=f"V row {row}")
        out, lse, rest = P.prompt_attention(q, k, v, rest=True, **at)
        spoilt = do.clone()
        spoilt[row, 3, 11] = BAD[bad]
        _, _, dv = P.prompt_attention_backward(spoilt, q, k, v, out, lse, rest=rest, **at)
        hit = torch.zeros_like(dv, dtype=torch.bool)
        hit[:row + 1, 1, 11] = True
        assert torch.equal(~torch.isfinite(dv), hit), row
        check(torch, dict(dv=torch.where(hit, want["dv"].to(dt), dv)), want, dt, d, what=f"d_out row {row}")
