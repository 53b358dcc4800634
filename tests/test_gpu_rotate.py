"""GPU parity of rotate_heads (adore_rotate_heads) and its gradients against the formulas in 64 bits.

Tolerances, with u = eps / 2 of the storage type, m the magnitude, and f = 2^-24 the rounding of fp32:
  sine and cosine: the angle is off by 2^-33 turns and two roundings of at most pi / 4 (1.6 f), the series' last addition by f / 2, the
  magnitude's product by f: less than 3 f; each product and the sum of a pair: f more.  So an element of a pair (a, b) is off by
  e = 4 f m (|a| + |b|) and its rounding, u (and f where that is another one) of itself.
  norms: a sum of 16 squares in a lane and of up to 8 lanes, at most 20 roundings, halved by the square root, and three more: r is off by
  13 f of itself, x r w by 15 f: 16 f (|a| + |b|) on top.
  gradients: g as above from d_out; the mean of w g x r by 48 f of the mean of sizes (its factors 28, its sums 20) and what e is off;
  dx = r (w g - x r mean) adds 32 f of either term.
  gradients of weights: sums of g x r, 30 f of a term, and 64 f of the sum of sizes for the additions (fewer than 64 one behind the other)."""
import math

import pytest

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
F = 2.0 ** -24
TINY = 2.0 ** -120


def _mods():
    import torch
    import paper_2407_02328_amd as P
    return torch, P


def draw(torch, shape, dtype, seed, std=1.0):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return torch.empty(shape, dtype=dtype, device=DEV).normal_(0.0, std, generator=g)


def dtype_of(torch, name):
    return torch.bfloat16 if name == "bf16" else torch.float32


def frequencies(torch, R, base=10000.0, factor=1.0, original=None, low=1.0, high=32.0):
    f = torch.tensor([base ** (-2.0 * j / R) for j in range(R // 2)], dtype=torch.float64, device=DEV)
    if original is None:
        return f / factor
    whole = ((original * f / (2 * math.pi) - low) / (high - low)).clamp(0, 1)
    return f * (whole + (1 - whole) / factor)


class Formula:
    """Rows [tokens][heads][d] at positions [tokens], in 64 bits."""

    def __init__(self, torch, positions, R, d, interleaved=False, magnitude=1.0, eps=1e-6, **scaled):
        self.torch, self.R, self.d, self.eps, self.m = torch, R, d, eps, magnitude
        i = torch.arange(R // 2, device=DEV)
        self.a, self.b = (2 * i, 2 * i + 1) if interleaved else (i, i + R // 2)
        if R:
            t = positions.double()[:, None] * frequencies(torch, R, **scaled)
            self.c, self.s = (magnitude * torch.cos(t))[:, None], (magnitude * torch.sin(t))[:, None]

    def turned(self, y, back=False):
        z = y.clone()
        if self.R:
            a, b, s = y[..., self.a], y[..., self.b], -self.s if back else self.s
            z[..., self.a], z[..., self.b] = a * self.c - b * s, a * s + b * self.c
        return z

    def pairs(self, y):
        """m (|a| + |b|) at both elements of a pair, |y| elsewhere."""
        z = y.abs()
        if self.R:
            s = self.m * (z[..., self.a] + z[..., self.b])
            z = z.clone()
            z[..., self.a], z[..., self.b] = s, s
        return z

    def size(self, x):
        return 1.0 / self.torch.sqrt(x.square().mean(-1, keepdim=True) + self.eps)

    def forward(self, x, w):
        x = x.double()
        y = x if w is None else x * self.size(x) * w.double()
        off = (4 if w is None else 20) * F * self.pairs(y)
        return self.turned(y), off

    def backward(self, d_out, x, w):
        g = self.turned(d_out.double(), back=True)
        off = 4 * F * self.pairs(d_out.double())
        if w is None:
            return g, off, None, None
        x, w = x.double(), w.double()
        r = self.size(x)
        n, wg = x * r, g * w
        dot = (wg * n).mean(-1, keepdim=True)
        dot_off = 48 * F * (wg * n).abs().mean(-1, keepdim=True) + ((w * off).abs() * n.abs()).mean(-1, keepdim=True)
        dx = r * (wg - n * dot)
        dx_off = r * ((w * off).abs() + 32 * F * wg.abs() + n.abs() * dot_off + 32 * F * (n * dot).abs())
        flat = lambda z: z.flatten(0, -2).sum(0)  # noqa: E731
        return dx, dx_off, flat(g * n), flat(off * n.abs()) + (30 + 64) * F * flat((g * n).abs())


def near(torch, got, want, off, dtype, what):
    u = torch.finfo(dtype).eps / 2
    bound = (u + (F if dtype != torch.float32 else 0.0)) * want.abs() + (1 + u) * off + TINY
    x = got.double()
    assert bool(((x - want).abs() <= bound).all()), f"{what}: worst {((x - want).abs() - bound).max().item()} of {want.abs().max().item()}"


def both_ways(torch, P, q, k, positions, f, rotary, dt, *, qw=None, kw=None, seed=9, flat=lambda x: x, **how):
    """Forward and backward of q and k (k may be None) against the formula; flat: the layout of a tensor to [tokens][heads][d]."""
    dqo = draw(torch, q.shape, dt, seed)
    dko = None if k is None else draw(torch, k.shape, dt, seed + 1)
    got = P.rotate_heads(q, k, positions, rotary, q_weight=qw, k_weight=kw, **how)
    grads = P.rotate_heads_backward(dqo, dko, q, k, positions, rotary, q_weight=qw, k_weight=kw, **how)
    for name, x, d_out, w, y, dx, dw in (("q", q, dqo, qw, got[0], grads[0], grads[2]), ("k", k, dko, kw, got[1], grads[1], grads[3])):
        if x is None:
            assert y is None and dx is None and dw is None
            continue
        near(torch, flat(y), *f.forward(flat(x), w), dt, name)
        want, off, want_w, off_w = f.backward(flat(d_out), flat(x), w)
        near(torch, flat(dx), want, off, dt, "d" + name)
        assert (dw is None) == (w is None)
        if w is not None:
            near(torch, dw, want_w, off_w, torch.float32, f"d{name}_weight")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("d,R", [(64, 64), (64, 16), (64, 48), (128, 128), (128, 96), (128, 32)])
def test_layouts_and_parts_of_the_head(d, R, interleaved, dtype):
    """Views of one projection, positions in any order."""
    torch, P = _mods()
    dt = dtype_of(torch, dtype)
    for T, H, Hk in ((1, 1, 1), (7, 4, 1), (33, 6, 2), (130, 3, 3)):
        qkv = draw(torch, (T, H + 2 * Hk, d), dt, T)
        pos = (torch.arange(T, device=DEV) * 7919 % 4099).int()
        f = Formula(torch, pos, R, d, interleaved)
        rotary = P.Rotary(R, interleaved=interleaved)
        both_ways(torch, P, qkv[:, :H], qkv[:, H:H + Hk], pos, f, rotary, dt)
        qw, kw = 1.0 + 0.3 * draw(torch, (d,), torch.float32, 3), 1.0 + 0.3 * draw(torch, (d,), torch.float32, 4)
        both_ways(torch, P, qkv[:, :H], qkv[:, H:H + Hk], pos, f, rotary, dt, qw=qw, kw=kw)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_norms_of_one_tensor_and_without_rotation(dtype):
    torch, P = _mods()
    dt = dtype_of(torch, dtype)
    q, k = draw(torch, (50, 4, 64), dt, 1, 3.0), draw(torch, (50, 2, 64), dt, 2, 0.01)
    pos = torch.arange(50, dtype=torch.int32, device=DEV)
    w = 1.0 + 0.5 * draw(torch, (64,), torch.float32, 3)
    f, none = Formula(torch, pos, 64, 64), Formula(torch, pos, 0, 64)
    rotary = P.Rotary(64)
    both_ways(torch, P, q, k, pos, f, rotary, dt, qw=w)
    both_ways(torch, P, q, k, pos, f, rotary, dt, kw=w)
    both_ways(torch, P, q, k, None, none, None, dt, qw=w)
    both_ways(torch, P, q, k, None, none, None, dt, qw=w, kw=w + 1.0)
    both_ways(torch, P, q, None, pos, f, rotary, dt)
    both_ways(torch, P, q, None, pos, f, rotary, dt, qw=w)
    g = Formula(torch, pos, 64, 64, eps=0.5)
    both_ways(torch, P, q, k, pos, g, rotary, dt, qw=w, kw=w, eps=0.5)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_dense_batches_and_strides(dtype):
    torch, P = _mods()
    dt = dtype_of(torch, dtype)
    B, H, Hk, S, d = 3, 5, 2, 41, 64
    flat = lambda x: x.transpose(1, 2).flatten(0, 1)  # noqa: E731
    q, k = draw(torch, (B, S, H, d + 16), dt, 1).transpose(1, 2)[..., 8:-8], draw(torch, (B, Hk, S, d), dt, 2)
    pos = torch.randint(0, 100000, (B, S), device=DEV, dtype=torch.int32)
    w = 1.0 + 0.5 * draw(torch, (d,), torch.float32, 3)
    rotary = P.Rotary(48)
    for p in (pos, pos[:1].expand(B, S), pos[0], pos.t().contiguous().t()):
        f = Formula(torch, p.expand(B, S).reshape(-1), 48, d)
        both_ways(torch, P, q, k, p, f, rotary, dt, flat=flat)
        both_ways(torch, P, q, k, p, f, rotary, dt, flat=flat, qw=w, kw=w)
    # a token of every sequence, positions out of another tensor's column
    cursor = torch.randint(0, 5000, (S, 3), device=DEV, dtype=torch.int32)
    x = draw(torch, (S, 4, d), dt, 5)
    both_ways(torch, P, x, x[:, :1], cursor[:, 1], Formula(torch, cursor[:, 1], 48, d), rotary, dt)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("scaled", [dict(factor=4.0), dict(factor=8.0, original=4096.0), dict(factor=32.0, original=2048.0, low=1.0, high=4.0, base=500000.0)])
def test_far_positions_and_scaled_frequencies(scaled, dtype):
    """As exact at 2^22 and below 0 as near 0; beyond, the reference's own angles lose too much (2^-53 of them)."""
    torch, P = _mods()
    dt = dtype_of(torch, dtype)
    pos = torch.tensor([0, 1, -1, 2, 3, 1000, -4097, 65535, 1 << 20, (1 << 22) - 1, -(1 << 22)], dtype=torch.int32, device=DEV)
    q, k = draw(torch, (len(pos), 3, 128), dt, 1), draw(torch, (len(pos), 1, 128), dt, 2)
    f = Formula(torch, pos, 128, 128, magnitude=1.25, **scaled)
    both_ways(torch, P, q, k, pos, f, P.Rotary(128, magnitude=1.25, **scaled), dt)


def test_the_largest_positions():
    """2^31 - 1 and -2^31 by exact arithmetic: the whole turns of position * turns / 2^64 are dropped in integers."""
    torch, P = _mods()
    rotary = P.Rotary(64)
    pos = [2 ** 31 - 1, -2 ** 31, 2 ** 30 + 12345]
    x = draw(torch, (3, 2, 64), torch.float32, 1)
    got, _ = P.rotate_heads(x, None, torch.tensor(pos, dtype=torch.int32, device=DEV), rotary)
    for i, p in enumerate(pos):
        t = torch.tensor([(p * (int(s) % (1 << 64)) % (1 << 64)) / 2.0 ** 64 * 2 * math.pi for s in rotary.turns], dtype=torch.float64, device=DEV)
        a, b = x[i].double().split(32, -1)
        want = torch.cat([a * t.cos() - b * t.sin(), a * t.sin() + b * t.cos()], -1)
        near(torch, got[i], want, 4 * F * torch.cat([a.abs() + b.abs()] * 2, -1), torch.float32, f"position {p}")


def test_as_the_library_turns_its_own_keys():
    """The reading that the oracle and rope_base have: halves, base^(-2j/d)."""
    import numpy as np
    from oracle.adore_oracle import rotary
    torch, P = _mods()
    x = draw(torch, (9, 2, 64), torch.bfloat16, 1)
    pos = [0, 1, 2, 77, 500, 501, 1023, 4000, 9215]
    got, _ = P.rotate_heads(x, None, torch.tensor(pos, dtype=torch.int32, device=DEV), P.Rotary(64, base=10000.0))
    want = torch.tensor(np.asarray(rotary(x.float().cpu().numpy(), pos, 10000.0)), device=DEV)
    a, b = x.double().abs().split(32, -1)
    near(torch, got, want, 4 * F * torch.cat([a + b] * 2, -1), torch.bfloat16, "oracle")


def test_many_tokens():
    """More than a launch has waves for at once, and sums of weights over all workgroups."""
    torch, P = _mods()
    for dt, d, T, H, Hk in ((torch.bfloat16, 128, 9001, 8, 2), (torch.float32, 64, 20011, 2, 1)):
        q, k = draw(torch, (T, H, d), dt, 1), draw(torch, (T, Hk, d), dt, 2)
        pos = torch.arange(T, dtype=torch.int32, device=DEV)
        w = 1.0 + 0.3 * draw(torch, (d,), torch.float32, 3)
        both_ways(torch, P, q, k, pos, Formula(torch, pos, d, d), P.Rotary(d), dt, qw=w, kw=w)


def test_in_place_and_into_places_of_one_tensor():
    torch, P = _mods()
    for dt in (torch.bfloat16, torch.float32):
        qkv = draw(torch, (77, 8, 64), dt, 1)
        q, k, v = qkv[:, :4], qkv[:, 4:6], qkv[:, 6:]
        pos = torch.arange(77, dtype=torch.int32, device=DEV)
        w = 1.0 + 0.3 * draw(torch, (64,), torch.float32, 3)
        rotary = P.Rotary(64)
        want = P.rotate_heads(q, k, pos, rotary, q_weight=w, k_weight=w)
        dq, dk = draw(torch, (77, 4, 64), dt, 5), draw(torch, (77, 2, 64), dt, 6)
        grads = P.rotate_heads_backward(dq, dk, q, k, pos, rotary, q_weight=w, k_weight=w)
        d_qkv = torch.full_like(qkv, 7.0)
        d_qkv[:, :4], d_qkv[:, 4:6] = dq, dk
        P.rotate_heads_backward(d_qkv[:, :4], d_qkv[:, 4:6], q, k, pos, rotary, q_weight=w, k_weight=w, dq=d_qkv[:, :4], dk=d_qkv[:, 4:6])
        assert torch.equal(d_qkv[:, :4], grads[0]) and torch.equal(d_qkv[:, 4:6], grads[1]) and bool((d_qkv[:, 6:] == 7.0).all())
        before = v.clone()
        got = P.rotate_heads(q, k, pos, rotary, q_weight=w, k_weight=w, q_out=q, k_out=k)
        assert got[0] is q and torch.equal(q, want[0]) and torch.equal(k, want[1]) and torch.equal(v, before)


@pytest.mark.parametrize("norm", [False, True])
def test_nothing_to_rotate(norm):
    torch, P = _mods()
    w = torch.ones(64, device=DEV) if norm else None
    for shape, kv in (((0, 4, 64), (0, 2, 64)), ((2, 4, 0, 64), (2, 2, 0, 64))):
        q, k = torch.empty(shape, device=DEV), torch.empty(kv, device=DEV)
        pos = torch.empty(shape[:1] if len(shape) == 3 else (2, 0), dtype=torch.int32, device=DEV)
        got = P.rotate_heads(q, k, pos, P.Rotary(64), q_weight=w, k_weight=w)
        assert got[0].shape == shape and got[1].shape == kv
        dq, dk, dqw, dkw = P.rotate_heads_backward(q, k, q, k, pos, P.Rotary(64), q_weight=w, k_weight=w)
        assert not norm or (bool((dqw == 0).all()) and bool((dkw == 0).all()))


def test_rows_that_are_not_finite_stay_among_themselves():
    torch, P = _mods()
    for dt in (torch.bfloat16, torch.float32):
        q = draw(torch, (40, 3, 64), dt, 1)
        pos = torch.arange(40, dtype=torch.int32, device=DEV)
        w = torch.ones(64, device=DEV)
        want = P.rotate_heads(q, q, pos, P.Rotary(64), q_weight=w)
        for bad in (math.nan, math.inf):
            x = q.clone()
            x[7, 1, 5] = bad
            x[20:] = bad
            got = P.rotate_heads(x, x, pos, P.Rotary(64), q_weight=w)
            dq, _, _, _ = P.rotate_heads_backward(q, q, x, x, pos, P.Rotary(64), q_weight=w)
            fine = torch.ones((40, 3), dtype=torch.bool, device=DEV)
            fine[7, 1], fine[20:] = False, False
            for a, b in zip(got, want):
                assert torch.equal(a[fine], b[fine])
            assert bool(torch.isfinite(dq[fine]).all()) and not bool(torch.isfinite(got[1][7, 1, 5])) and bool(torch.isfinite(got[1][7, 1, 6]))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("interleaved", [False, True])
def test_what_is_not_turned_stays_as_it_is(interleaved, dtype):
    """Elements behind the turned part come through to the bit, and what is not finite among them reaches no other element."""
    torch, P = _mods()
    dt = dtype_of(torch, dtype)
    for d, R in ((64, 16), (64, 48), (128, 32), (128, 96)):
        q = draw(torch, (9, 2, d), dt, 1)
        pos = torch.arange(9, dtype=torch.int32, device=DEV)
        rotary = P.Rotary(R, interleaved=interleaved, magnitude=1.5)
        want, _ = P.rotate_heads(q, None, pos, rotary)
        assert torch.equal(want[..., R:], q[..., R:])
        back = P.rotate_heads_backward(q, None, q, None, pos, rotary)[0]
        assert torch.equal(back[..., R:], q[..., R:])
        for bad in (math.inf, math.nan):
            for e in (R, d - 1, (R + d) // 2):
                x = q.clone()
                x[4, 1, e] = bad
                got, _ = P.rotate_heads(x, None, pos, rotary)
                grad = P.rotate_heads_backward(x, None, q, None, pos, rotary)[0]
                for y, z in ((got, want), (grad, back)):
                    other = torch.ones_like(y, dtype=torch.bool)
                    other[4, 1, e] = False
                    assert torch.equal(y[other], z[other]) and not bool(torch.isfinite(y[4, 1, e]))


def test_gradients_against_differences():
    """Central differences in 64 bits of the fp32 outputs: h = 2^-6 leaves h^2 / 6 of the third derivative, and rounding 2^-24 sqrt(n) / h."""
    torch, P = _mods()
    q, k = draw(torch, (30, 4, 64), torch.float32, 1), draw(torch, (30, 2, 64), torch.float32, 2)
    qw, kw = (1.0 + 0.3 * draw(torch, (64,), torch.float32, s) for s in (3, 4))
    dq, dk = draw(torch, q.shape, torch.float32, 5), draw(torch, k.shape, torch.float32, 6)
    pos = torch.arange(30, dtype=torch.int32, device=DEV) * 3
    rotary = P.Rotary(32, interleaved=True, magnitude=1.1)

    def loss(a, b, c, e):
        x, y = P.rotate_heads(a, b, pos, rotary, q_weight=c, k_weight=e)
        return float((x.double() * dq.double()).sum() + (y.double() * dk.double()).sum())

    args = [q, k, qw, kw]
    grads = P.rotate_heads_backward(dq, dk, q, k, pos, rotary, q_weight=qw, k_weight=kw)
    h = 2.0 ** -6
    for i, x in enumerate(args):
        u = draw(torch, x.shape, torch.float32, 50 + i)
        hi, lo = list(args), list(args)
        hi[i], lo[i] = x + h * u, x - h * u
        slope = (loss(*hi) - loss(*lo)) / (2 * h)
        want = float((grads[i].double() * u.double()).sum())
        size = float((grads[i].double() * u.double()).square().sum().sqrt())
        assert abs(slope - want) < 0.02 * size + 1e-3, (i, slope, want, size)


def test_autograd():
    torch, P = _mods()
    for dt in (torch.bfloat16, torch.float32):
        leaves = [draw(torch, (20, 8, 64), dt, 1).requires_grad_(), *((1.0 + 0.3 * draw(torch, (64,), torch.float32, s)).requires_grad_() for s in (3, 4))]
        x, qw, kw = leaves
        pos = torch.arange(20, dtype=torch.int32, device=DEV)
        rotary = P.Rotary(64)
        q, k = P.rotate_heads(x[:, :4], x[:, 4:6], pos, rotary, q_weight=qw, k_weight=kw)
        dq, dk = draw(torch, q.shape, dt, 5), draw(torch, k.shape, dt, 6)
        torch.autograd.backward([q, k], [dq, dk])
        want = P.rotate_heads_backward(dq, dk, x.detach()[:, :4], x.detach()[:, 4:6], pos, rotary, q_weight=qw.detach(), k_weight=kw.detach())
        assert torch.equal(x.grad[:, :4], want[0]) and torch.equal(x.grad[:, 4:6], want[1]) and bool((x.grad[:, 6:] == 0).all())
        assert torch.equal(qw.grad, want[2]) and torch.equal(kw.grad, want[3])
        # only one of the results goes on: the other's gradient is zeros; a gradient of any layout
        y = x.detach().clone().requires_grad_()
        q, _ = P.rotate_heads(y[:, :4], y[:, 4:6], pos, rotary)
        q.sum().backward()
        ones = torch.ones_like(dq)
        assert torch.equal(y.grad[:, :4], P.rotate_heads_backward(ones, None, y.detach()[:, :4], None, pos, rotary)[0])
        assert bool((y.grad[:, 4:] == 0).all())
        z = x.detach()[:, :4].clone().requires_grad_()
        only, none = P.rotate_heads(z, None, pos, rotary, q_weight=qw.detach())
        assert none is None
        only.backward(dq)
        assert torch.equal(z.grad, want[0])
        alone = kw.detach().clone().requires_grad_()             # a weight's gradient, the rows have none
        _, k = P.rotate_heads(x.detach()[:, :4], x.detach()[:, 4:6], pos, rotary, k_weight=alone)
        k.backward(dk)
        assert torch.equal(alone.grad, want[3])
        with pytest.raises(ValueError):
            P.rotate_heads(y[:, :4], None, pos, rotary, q_out=torch.empty_like(dq))


def test_equal_inputs_give_equal_bits_and_a_graph_replays():
    torch, P = _mods()
    q, k = draw(torch, (500, 8, 128), torch.bfloat16, 1), draw(torch, (500, 2, 128), torch.bfloat16, 2)
    dq, dk = draw(torch, q.shape, torch.bfloat16, 3), draw(torch, k.shape, torch.bfloat16, 4)
    w = 1.0 + 0.3 * draw(torch, (128,), torch.float32, 5)
    pos = torch.arange(500, dtype=torch.int32, device=DEV)
    rotary = P.Rotary(128)

    def all_of_it():
        return (*P.rotate_heads(q, k, pos, rotary, q_weight=w, k_weight=w),
                *P.rotate_heads_backward(dq, dk, q, k, pos, rotary, q_weight=w, k_weight=w))

    want = [x.clone() for x in all_of_it()]
    for x, y in zip(all_of_it(), want):
        assert torch.equal(x, y)
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        for x, y in zip(all_of_it(), want):        # (on another stream than the default)
            assert torch.equal(x, y)
    torch.cuda.current_stream().wait_stream(stream)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = all_of_it()
    for turn in range(3):
        for x in got:
            x.fill_(3.0)
        pos.add_(turn * 11)
        graph.replay()
        torch.cuda.synchronize()
        for x, y in zip(got, all_of_it()):
            assert torch.equal(x, y), turn
