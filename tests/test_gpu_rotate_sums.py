"""Gradients of the norms' weights over very many rows: sums that a lane makes of its rows one after the other are taken over at every 64th, so
that what additions lose does not grow with the rows.

Tolerance: with f = 2^-24, a term is off by 30 f of itself (test_gpu_rotate.py).  Rows r are shared by 16384 groups of lanes at 128 elements and by
32768 at 64 (512 workgroups of four waves): up to 64 additions one behind the other, n = r / 64 of the groups' rows for those, 8 for lanes and
waves, 16 and 5 for workgroups.  All terms of an element here are the same: (30 + 64 + n + 29) f of their sum."""
import pytest

from tests.test_gpu_rotate import DEV, F, _mods, draw, dtype_of

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,d,tokens,heads", [("bf16", 128, 1 << 20, 32), ("f32", 64, (1 << 20) + 77, 40)])
def test_many_equal_rows(dtype, d, tokens, heads):
    """One row and one gradient, read by all tokens and heads (strides of 0), so that every addition of an element is rounded the same way."""
    torch, P = _mods()
    dt = dtype_of(torch, dtype)
    x, g = draw(torch, (d,), dt, 1), draw(torch, (d,), dt, 2)
    w = 1.0 + 0.3 * draw(torch, (d,), torch.float32, 3)
    rows = lambda y: y.expand(tokens, heads, d)  # noqa: E731
    _, _, dw, _ = P.rotate_heads_backward(rows(g), None, rows(x), None, None, None, q_weight=w)
    term = g.double() * x.double() / (x.double().square().mean() + 1e-6).sqrt()
    n = -(-tokens * heads // (16384 if d == 128 else 32768)) // 64 + 1
    off = (dw.double() - tokens * heads * term).abs() / (tokens * heads * term.abs())
    assert float(off.max()) <= (30 + 64 + n + 29) * F, f"worst {float(off.max()) / F} of 2^-24"
