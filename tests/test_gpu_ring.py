"""GPU parity of the window cache (adore_ring_fill, adore_ring_step, adore_ring_read) against its definition in 64 bits: a sequence's
history, of which the first `sinks` and the last `window` tokens are seen.

What it holds, its order and positions are exact.  Outputs, with u = eps / 2 of the storage type and t = 2^-24 (d max(scale sum |q| |k|) + 8
+ slots) what a weight's exponent and the sum of all weights are off by (fp32 sums):
  u |out| + (t + term) sum p |v|      term: 2^-16 bf16 (a weight in two terms), 2^-22 fp32"""
import math

import numpy as np
import pytest

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def _mods():
    import torch
    import paper_2407_02328_amd as P
    return torch, P


def draw(torch, shape, dtype, seed, std=1.0):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return torch.empty(shape, dtype=dtype, device=DEV).normal_(0.0, std, generator=g)


class History:
    """All rows that a sequence has had, 64 bits: k, v [tokens][Hk][d]."""

    def __init__(self, torch, P, B, H, Hk, d, window, sinks, dtype, scale=None, **buffers):
        self.torch, self.B, self.H, self.Hk, self.d, self.W, self.S, self.scale = torch, B, H, Hk, d, window, sinks, scale or d ** -0.5
        self.dt = torch.bfloat16 if dtype == "bf16" else torch.float32
        self.cache = P.WindowCache(batch=B, heads=H, kv_heads=Hk, head_dim=d, window=window, sinks=sinks, dtype=dtype, scale=scale, **buffers)
        none = torch.zeros((0, Hk, d), dtype=torch.float64, device=DEV)
        self.k, self.v = [none] * B, [none] * B

    def kept(self, x):
        return x if len(x) <= self.S + self.W else self.torch.cat([x[:self.S], x[len(x) - self.W:]])

    def fill(self, lengths, seed, dense=False):
        torch = self.torch
        if dense:
            kv = draw(torch, (self.B, 2 * self.Hk, lengths[0], self.d), self.dt, seed)
            k, v = kv[:, :self.Hk], kv[:, self.Hk:]
            self.cache.fill(k, v)
            self.k, self.v = ([x.transpose(0, 1).double() for x in y] for y in (k, v))
            return
        T = sum(lengths) + 2
        kv = draw(torch, (T, 2 * self.Hk, self.d), self.dt, seed)
        k, v = kv[:, :self.Hk], kv[:, self.Hk:]
        start = np.cumsum([1] + list(lengths))
        self.cache.fill(k, v, k_start=torch.tensor(start, dtype=torch.int32, device=DEV))
        self.k, self.v = ([x[a:b].double() for a, b in zip(start, start[1:])] for x in (k, v))

    def step(self, seed, std=1.0, spoil=None):
        torch = self.torch
        q, k, v = draw(torch, (self.B, self.H, self.d), self.dt, seed, std), draw(torch, (self.B, self.Hk, self.d), self.dt, seed + 1), \
            draw(torch, (self.B, self.Hk, self.d), self.dt, seed + 2)
        if spoil:
            spoil(q, k, v)
        out = self.cache.step(q, k, v)
        u, g = torch.finfo(self.dt).eps / 2, self.H // self.Hk
        for b in range(self.B):
            self.k[b], self.v[b] = torch.cat([self.k[b], k[b:b + 1].double()]), torch.cat([self.v[b], v[b:b + 1].double()])
            kk, vv = (self.kept(x).permute(1, 0, 2).contiguous() for x in (self.k[b], self.v[b]))      # [Hk][n][d]
            qq, kt = q[b].double().view(self.Hk, g, self.d), kk.transpose(1, 2).contiguous()
            p = torch.softmax(qq @ kt * self.scale, -1)
            size = float(torch.nan_to_num(qq.abs() @ kt.abs(), nan=0.0, posinf=0.0).amax()) * self.scale      # (of heads that have numbers)
            t = 2.0 ** -24 * (self.d * size + 8 + self.W + self.S) + (2.0 ** -16 if self.dt == torch.bfloat16 else 2.0 ** -22)
            want, bound = (p @ vv).view(self.H, self.d), (p @ vv.abs()).view(self.H, self.d)
            x = out[b].double()
            fine = torch.isfinite(want)
            assert torch.equal(torch.isfinite(x), fine), f"sequence {b}: {int((torch.isfinite(x) != fine).sum())} elements"
            off = (x - want).abs() - (u * want.abs() + t * bound)
            assert bool((off[fine] <= 0).all()), f"sequence {b}: worst {off[fine].max().item()}"

    def compare(self):
        torch = self.torch
        k, v = self.cache.read()
        for b in range(self.B):
            for got, rows in ((k[b], self.k[b]), (v[b], self.v[b])):
                want = self.kept(rows).transpose(0, 1)
                assert torch.equal(got[:, :want.shape[1]].double(), want), b
                assert bool((got[:, want.shape[1]:] == 0).all()), b
            assert bool((self.cache.cursor[b] == len(self.k[b])).all())
        assert self.cache.positions.tolist() == [len(x) for x in self.k]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 1), (7, 0), (31, 1), (32, 0), (33, 31), (100, 4), (5, 70)])
def test_from_nothing_until_it_has_gone_round(window, sinks, d, dtype):
    torch, P = _mods()
    h = History(torch, P, 2, 6, 2, d, window, sinks, dtype)
    h.compare()
    for n in range(min(2 * window + sinks + 3, 150)):
        h.step(100 + 3 * n)
        if n % 7 == 0:
            h.compare()
    h.compare()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("B,H,Hk,d,window,sinks", [(5, 4, 4, 64, 60, 4), (5, 8, 1, 128, 128, 0), (5, 20, 1, 64, 200, 9), (5, 48, 1, 128, 65, 2), (5, 6, 3, 64, 1, 3),
                                                   (5, 16, 16, 64, 3, 0)])
def test_prompts_of_all_lengths(B, H, Hk, d, window, sinks, dtype):
    """Empty and short ones, full ones, and those that have gone round more than once; groups of more than 16 heads."""
    torch, P = _mods()
    slots = window + sinks
    h = History(torch, P, B, H, Hk, d, window, sinks, dtype)
    for seed, lengths in enumerate(([0, 1, sinks, slots, slots + 1], [slots - 1, 2 * slots + 5, 3 * window + sinks, slots + window, 17], [5, 0, 900, 33, 64])):
        h.fill(lengths, seed)
        h.compare()
        for n in range(4):
            h.step(1000 * seed + 3 * n)
        h.compare()
    h.fill([77] * B, 50, dense=True)
    h.compare()
    h.step(60)
    h.compare()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("B,H,Hk,d,window,sinks,tokens", [(1, 8, 2, 128, 5000, 4, 20000), (2, 4, 1, 64, 3000, 50, 2900), (3, 40, 2, 64, 2048, 0, 4100), (1, 1, 1, 64, 9000, 1, 8000)])
def test_rows_that_workgroups_share(B, H, Hk, d, window, sinks, tokens, dtype):
    torch, P = _mods()
    h = History(torch, P, B, H, Hk, d, window, sinks, dtype)
    h.fill([tokens - 700 * b for b in range(B)], 1)
    h.compare()
    for n in range(3):
        h.step(10 + 3 * n, std=4.0 if n == 2 else 1.0)
    h.compare()


@pytest.mark.parametrize("std,scale", [(30.0, None), (1e-4, None), (1.0, 2.0)])
def test_sharp_and_flat_weights(std, scale):
    torch, P = _mods()
    for dtype in ("bf16", "f32"):
        h = History(torch, P, 2, 4, 2, 64, 300, 4, dtype, scale=scale)
        h.fill([500, 200], 1)
        for n in range(3):
            h.step(10 + 3 * n, std=std)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("window,sinks,tokens", [(40, 3, 100), (3000, 2, 5000)])
def test_rows_that_have_left_may_have_held_anything(window, sinks, tokens, dtype):
    """NaN and infinities in free slots, in the row that the token takes, and in rows of the window, which reach their own heads only."""
    torch, P = _mods()
    h = History(torch, P, 2, 4, 2, 64, window, sinks, dtype)
    h.cache.cache.fill_(math.nan)
    for n in range(3):
        h.step(3 * n)                       # free slots are not read
    h.cache.cache.fill_(math.inf)
    h.fill([tokens, 5], 1)

    def spoil(q, k, v):
        k[0, 1], v[0, 1] = math.nan, math.nan

    h.step(20, spoil=spoil)
    for n in range(3):
        h.step(30 + 3 * n)                  # kv head 1 of sequence 0 is spoilt, the others are not
    if window == 40:
        for n in range(60):
            h.step(100 + 3 * n)             # it has left: nothing of it is there
        assert all(bool(torch.isfinite(h.cache.read()[i]).all()) for i in (0, 1))


def test_rows_in_between_that_were_left_out():
    """read(), new rows behind it, fill() with how many tokens there have been: as if all had been there."""
    torch, P = _mods()
    for dtype in ("bf16", "f32"):
        h = History(torch, P, 2, 4, 2, 64, 50, 6, dtype)
        h.fill([333, 200], 1)
        k, v = h.cache.read()
        new = draw(torch, (2, 4, 23, 64), h.dt, 7)
        k, v = torch.cat([k, new[:, :2]], 2), torch.cat([v, new[:, 2:]], 2)
        h.cache.fill(k, v, seen=torch.tensor([356, 223], dtype=torch.int32, device=DEV))
        for b in range(2):
            h.k[b], h.v[b] = torch.cat([h.k[b], new[b, :2].transpose(0, 1).double()]), torch.cat([h.v[b], new[b, 2:].transpose(0, 1).double()])
        h.compare()
        for n in range(60):
            h.step(10 + 3 * n)
        h.compare()
        # fewer rows than slots: all there have been, whatever is said
        few = draw(torch, (2, 4, 9, 64), h.dt, 8)
        h.cache.fill(few[:, :2], few[:, 2:], seen=torch.tensor([500, 3], dtype=torch.int32, device=DEV))
        assert h.cache.positions.tolist() == [9, 9]


def test_buffers_of_the_callers_and_a_graph():
    torch, P = _mods()
    for dtype, window in (("bf16", 45), ("f32", 45), ("bf16", 4000)):
        dt = torch.bfloat16 if dtype == "bf16" else torch.float32
        shape = (2, 2, (window + 4 + 31) // 32, 64 * 64)
        ring, cursor = torch.zeros(shape, dtype=dt, device=DEV), torch.zeros((2, 2), dtype=torch.int32, device=DEV)
        make = lambda a, b: P.WindowCache(batch=2, heads=4, kv_heads=2, head_dim=64, window=window, sinks=4, dtype=dt, cache=a, cursor=b)  # noqa: E731
        captured, eager = make(ring, cursor), make(ring.clone(), cursor.clone())
        prompt = draw(torch, (2, 4, 60, 64), dt, 1)
        q, k, v = draw(torch, (2, 4, 64), dt, 2), draw(torch, (2, 2, 64), dt, 3), draw(torch, (2, 2, 64), dt, 4)
        stream = torch.cuda.Stream()
        stream.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(stream):
            captured.step(q, k, v)
        torch.cuda.current_stream().wait_stream(stream)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            out = captured.step(q, k, v)
        for c in (captured, eager):
            c.fill(prompt[:, :2], prompt[:, 2:])
        for n in range(70):
            for x, s in ((q, 10), (k, 11), (v, 12)):
                x.copy_(draw(torch, x.shape, dt, 100 * n + s))
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(out, eager.step(q, k, v)), n
        assert torch.equal(ring, eager.cache) and torch.equal(cursor, eager.cursor)


def test_a_step_writes_its_own_row_and_nothing_else():
    torch, P = _mods()
    for dt in (torch.bfloat16, torch.float32):
        c = P.WindowCache(batch=3, heads=4, kv_heads=2, head_dim=64, window=70, sinks=5, dtype=dt)
        kv = draw(torch, (3, 4, 200, 64), dt, 1)
        c.fill(kv[:, :2], kv[:, 2:])
        before = c.cache.clone()
        k, v = draw(torch, (3, 2, 64), dt, 3) + 10.0, draw(torch, (3, 2, 64), dt, 4) + 10.0
        c.step(draw(torch, (3, 4, 64), dt, 2), k, v)
        assert int((c.cache != before).sum()) == 3 * 2 * 2 * 64
        rk, rv = c.read()
        assert torch.equal(rk[:, :, -1], k) and torch.equal(rv[:, :, -1], v)


def test_offsets_beyond_32_bits():
    """A row of 2^20 slots of 128 elements in fp32 is 2^30 bytes: the last of 5 begins behind 2^32 bytes, the cache's elements pass 2^30."""
    torch, P = _mods()
    if torch.cuda.mem_get_info()[0] < 40 << 30:
        pytest.skip("not enough memory")
    c = P.WindowCache(batch=5, heads=2, kv_heads=1, head_dim=128, window=(1 << 20) - 4, sinks=4, dtype="f32")
    c.cursor.fill_(1 << 20)
    c.cursor[4] = (1 << 20) - 1                      # the last sequence's last slot is free
    kv = torch.zeros((5, 1, 128), device=DEV)
    q = torch.ones((5, 2, 128), device=DEV)
    k, v = kv + 1.0, kv + torch.arange(5, device=DEV)[:, None, None]
    out = c.step(q, k, v)
    # one row with weight e^{128 / sqrt(128)} among 2^20 of weight 1
    w = math.exp(128 ** 0.5)
    want = w * torch.arange(5, dtype=torch.float64, device=DEV) / (w + (1 << 20) - 1)
    # (exponents within 2^-24 (128 * 11.4 + 8), sums of 2^20 terms in fp32: at most 2^-24 * 2^20 / 256 one behind the other, both sides)
    assert bool(((out.double() - want[:, None, None]).abs() <= want[:, None, None] * 5e-4).all())
    rk, rv = c.read()
    assert bool((rk[4, 0, -1] == 1).all()) and bool((rv[4, 0, -1] == 4).all()) and bool((rk[4, 0, :-1] == 0).all())
