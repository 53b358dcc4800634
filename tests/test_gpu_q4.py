"""GPU parity of the cache held in 4 bits (adore_q4_fill, adore_q4_step, adore_q4_read) against its definition in 64 bits.

What it holds, which tokens stay and which slot comes next are exact.  Scores and outputs, with u = eps / 2 of the storage type and
t = 2^-24 (d max(scale sum |q| |k|) + 8 + slots) what a weight's exponent and the sum of all weights are off by (fp32 sums):
  out     u |out| + (t + term) sum p |v|      term: 2^-16 bf16 (a weight in two terms), 2^-22 fp32 (in three)
  score   what a step adds: 2 t of it, and a rounding of the sum, 2^-24.
The GPU's scores are checked and then taken over, so that the next step starts from the same bits on both sides; where two scores
that decide are within what they may be off by, both slots are right."""
import math

import numpy as np
import pytest

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
GRID = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def _mods():
    import torch
    import paper_2407_02328_amd as P
    return torch, P


def held_values(x):
    """Rows (64 bits, of storage values) as the cache holds them."""
    x = np.nan_to_num(np.asarray(x, dtype=np.float64), nan=0.0, posinf=2.0 ** 200, neginf=-2.0 ** 200)
    g = x.reshape(-1, 32)
    big = np.abs(g).max(1)
    _, e = np.frexp(big)                              # big = m 2^e, m in [0.5, 1)
    e = np.where(big > 0.875 * np.exp2(e.astype(float)), e - 2, e - 3)
    e = np.clip(np.where(big == 0, -100, e), -100, 125)
    y = np.minimum(np.abs(g) / np.exp2(e)[:, None], 8.0)       # (all distances from 2^75 are one number)
    far = np.abs(y[..., None] - GRID)
    best = far.min(-1, keepdims=True)
    near = far == best
    code = np.where(near & (np.arange(8) % 2 == 0), np.arange(8), 99).min(-1)          # the even one of two
    code = np.where(code == 99, near.argmax(-1), code)
    return (np.sign(g) * GRID[code] * np.exp2(e)[:, None]).reshape(x.shape)


def host(t):
    return t.detach().cpu().double().numpy() if t.dtype.is_floating_point else t.detach().cpu().numpy()


def draw(torch, shape, dtype, seed, std=1.0):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return torch.empty(shape, dtype=dtype, device=DEV).normal_(0.0, std, generator=g)


class Model:
    """The cache by its definition: values in 64 bits, one row (sequence, kv head) at a time."""

    def __init__(self, B, H, Hk, d, K, recent, scale=None):
        self.B, self.H, self.Hk, self.d, self.K, self.recent, self.scale = B, H, Hk, d, K, recent, scale or d ** -0.5
        self.k, self.v = np.zeros((B, Hk, K, d)), np.zeros((B, Hk, K, d))
        self.pos = np.full((B, Hk, K), -1)
        self.score = np.zeros((B, Hk, K), dtype=np.float32)
        self.cursor = np.zeros((B, Hk, 2), dtype=np.int64)

    def next_slot(self, pos, score, n, slack=0.0):
        """Right answers for the slot that token n takes."""
        free = np.flatnonzero(pos < 0)
        if len(free):
            return [int(free[0])]
        may = np.flatnonzero(pos < n - self.recent)
        s = score[may].astype(np.float64)
        return [int(x) for x in may[s <= s.min() + slack]][:1 if slack == 0.0 else None]

    def fill(self, lengths, rows_k, rows_v, scores):
        """rows_k[b] [n][Hk][d], scores[b] [Hk][n]."""
        for b, n in enumerate(lengths):
            for h in range(self.Hk):
                sc = scores[b][h].astype(np.float32)
                old = max(0, n - self.recent)
                goes = np.lexsort((np.arange(old), sc[:old]))[:max(0, n - self.K)]
                stay = np.setdiff1d(np.arange(n), goes)
                m = len(stay)
                self.k[b, h], self.v[b, h] = 0.0, 0.0
                self.k[b, h, :m], self.v[b, h, :m] = held_values(rows_k[b][stay, h]), held_values(rows_v[b][stay, h])
                self.pos[b, h], self.score[b, h] = -1, 0.0
                self.pos[b, h, :m], self.score[b, h, :m] = stay, sc[stay]
                self.cursor[b, h] = self.next_slot(self.pos[b, h], self.score[b, h], n)[0], n

    def step(self, q, k, v):
        """Out, its bound's sum, what every slot receives, and the exponents' size."""
        out, size_v, got, size = np.zeros((self.B, self.H, self.d)), np.zeros((self.B, self.H, self.d)), np.zeros(self.score.shape), 0.0
        g = self.H // self.Hk
        for b in range(self.B):
            for h in range(self.Hk):
                s, n = self.cursor[b, h]
                self.k[b, h, s], self.v[b, h, s] = held_values(k[b, h]), held_values(v[b, h])
                self.pos[b, h, s], self.score[b, h, s] = n, 0.0
                there = np.flatnonzero(self.pos[b, h] >= 0)
                kk, vv = self.k[b, h, there], self.v[b, h, there]
                qq = q[b, h * g:(h + 1) * g]
                w = qq @ kk.T * self.scale
                size = max(size, (np.abs(qq) @ np.abs(kk).T).max() * self.scale)
                p = np.exp(w - w.max(1, keepdims=True))
                p /= p.sum(1, keepdims=True)
                out[b, h * g:(h + 1) * g], size_v[b, h * g:(h + 1) * g] = p @ vv, p @ np.abs(vv)
                got[b, h, there] = p.sum(0)
        return out, size_v, got, size


def compare(torch, cache, m, what):
    k, v = (host(x) for x in cache.read())
    for name, x, y in (("k", k, m.k), ("v", v, m.v), ("slot_pos", host(cache.slot_pos), m.pos), ("cursor", host(cache.cursor), m.cursor),
                       ("score", host(cache.score).astype(np.float32), m.score)):
        assert np.array_equal(x, y), f"{what}: {name}, {(x != y).sum()} of {x.size} differ"


def take_step(torch, cache, m, dt, seed, what, q_std=1.0):
    q, k, v = draw(torch, (m.B, m.H, m.d), dt, seed, q_std), draw(torch, (m.B, m.Hk, m.d), dt, seed + 1), draw(torch, (m.B, m.Hk, m.d), dt, seed + 2)
    out, k_held, v_held = cache.step(q, k, v, held=True)
    assert np.array_equal(host(k_held), held_values(host(k))) and np.array_equal(host(v_held), held_values(host(v))), what
    want, size_v, got, size = m.step(host(q), host(k), host(v))
    u = torch.finfo(dt).eps / 2
    t = 2.0 ** -24 * (m.d * size + 8 + m.K)
    term = 2.0 ** -16 if dt == torch.bfloat16 else 2.0 ** -22
    off = np.abs(host(out) - want) - (u * np.abs(want) + (t + term) * size_v)
    assert off.max() <= 2.0 ** -120, f"{what}: out off by {off.max()} more"
    score = host(cache.score)
    bound = 2 * t * got + 2.0 ** -24 * (m.score + got) + 2.0 ** -120
    worst = (np.abs(score - (m.score.astype(np.float64) + got)) - bound).max()
    assert worst <= 0, f"{what}: score off by {worst} more"
    cursor = host(cache.cursor)
    for b in range(m.B):
        for h in range(m.Hk):
            n = m.cursor[b, h, 1] + 1
            right = m.next_slot(m.pos[b, h], m.score[b, h] + got[b, h], n, 2 * bound[b, h].max())
            assert cursor[b, h, 0] in right and cursor[b, h, 1] == n, (what, b, h, cursor[b, h], right, n)
    m.score, m.cursor = score.astype(np.float32), cursor.astype(np.int64)


def made(torch, P, B, H, Hk, d, K, recent, dt, lengths, seed=1, tied=False, scale=None):
    """A cache filled with prompts, and its model."""
    cache = P.Q4Cache(batch=B, heads=H, kv_heads=Hk, head_dim=d, slots=K, recent=recent, dtype=dt, scale=scale)
    m = Model(B, H, Hk, d, K, recent, scale)
    T = sum(lengths)
    k, v = draw(torch, (T, Hk, d), dt, seed), draw(torch, (T, Hk, d), dt, seed + 1)
    scores = draw(torch, (Hk, T), torch.float32, seed + 2).abs()
    if tied:
        scores = (scores * 2).round() / 2
    at = np.cumsum([0] + list(lengths))
    cache.fill(k, v, scores, k_start=torch.tensor(at, dtype=torch.int32, device=DEV))
    part = [slice(at[b], at[b + 1]) for b in range(B)]
    m.fill(lengths, [host(k)[p] for p in part], [host(v)[p] for p in part], [host(scores)[:, p] for p in part])
    return cache, m


def types():
    import torch
    return {"bf16": torch.bfloat16, "f32": torch.float32}


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("K,recent,lengths", [
    (2, 1, [0, 1, 2, 3]), (24, 5, [0, 1, 23, 24, 25, 100]), (63, 62, [62, 63, 64, 300]), (64, 1, [64, 65, 1500]), (65, 32, [64, 66, 2100]), (200, 13, [5, 1025, 199])])
def test_prompts_fill_the_cache(K, recent, lengths, d, dtype):
    torch, P = _mods()
    for tied in (False, True):
        cache, m = made(torch, P, len(lengths), 2, 2, d, K, recent, types()[dtype], lengths, tied=tied)
        compare(torch, cache, m, f"tied {tied}")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_a_dense_batch_without_scores_keeps_the_last_tokens(dtype):
    torch, P = _mods()
    dt = types()[dtype]
    cache = P.Q4Cache(batch=2, heads=3, kv_heads=3, head_dim=64, slots=20, recent=4, dtype=dt)
    k, v = draw(torch, (2, 3, 50, 64), dt, 1), draw(torch, (2, 50, 3, 64), dt, 2).transpose(1, 2)
    cache.fill(k, v)
    got_k, got_v = cache.read()
    assert bool((cache.slot_pos == torch.arange(30, 50, device=DEV)).all())
    assert np.array_equal(host(got_k), held_values(host(k[:, :, 30:]))) and np.array_equal(host(got_v), held_values(host(v[:, :, 30:])))
    assert bool((cache.cursor == torch.tensor([0, 50], device=DEV)).all())


def test_values_at_the_borders_of_the_format():
    """Ties between neighbouring codes, the largest element around 7 units, tiny and huge groups, zeros, infinities and NaN."""
    torch, P = _mods()
    units = [0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.0, 6.99, 7.0, 0.24, 0.26, 4.999, 5.001, 3.499, 0.0]
    for dt in types().values():
        for power in (-126, -110, -99, -98, -97, -3, 0, 7, 100, 124, 125):
            rows = torch.tensor([[x * s for x in units for s in (1.0, -1.0)] for _ in range(6)], dtype=torch.float64)
            rows[1, 0], rows[2, 0], rows[3, 0], rows[4, :], rows[5, 5] = 3.51, 7.01, math.nan, 0.0, math.inf
            rows = (rows * 2.0 ** power).clamp(-3.3e38, 3.3e38)
            rows[5, 5] = math.inf
            x = rows.to(dt).repeat(1, 2)[:, None].contiguous().to(DEV)               # [6][1][64]
            cache = P.Q4Cache(batch=1, heads=1, kv_heads=1, head_dim=64, slots=6, recent=1, dtype=dt)
            cache.fill(x, x.flip(0).contiguous(), k_start=torch.tensor([0, 6], dtype=torch.int32, device=DEV))
            k, v = cache.read()
            want = held_values(host(x))[:, 0]
            assert np.array_equal(host(k)[0, 0], want), (dt, power)
            assert np.array_equal(host(v)[0, 0], want[::-1]), (dt, power)
            again = P.Q4Cache(batch=1, heads=1, kv_heads=1, head_dim=64, slots=6, recent=1, dtype=dt)
            q = torch.zeros((1, 1, 64), dtype=dt, device=DEV)
            for i in range(6):
                again.step(q, x[i][None].contiguous(), x[5 - i][None].contiguous())
            k, v = again.read()
            assert np.array_equal(host(k)[0, 0], want) and np.array_equal(host(v)[0, 0], want[::-1]), (dt, power)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("H,Hk,d", [(1, 1, 64), (4, 4, 128), (8, 2, 128), (5, 1, 128), (16, 1, 128), (17, 1, 128), (24, 3, 64), (9, 1, 64), (40, 1, 64), (7, 7, 64)])
def test_steps(H, Hk, d, dtype):
    torch, P = _mods()
    for K, recent, lengths in ((70, 9, [3, 69, 200]), (130, 1, [130, 0])):
        cache, m = made(torch, P, len(lengths), H, Hk, d, K, recent, types()[dtype], lengths)
        for i in range(6):
            take_step(torch, cache, m, types()[dtype], 100 + 10 * i, f"K {K} step {i}")
        compare(torch, cache, m, f"K {K}")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_from_an_empty_cache_until_it_evicts(dtype):
    torch, P = _mods()
    dt = types()[dtype]
    cache = P.Q4Cache(batch=2, heads=4, kv_heads=2, head_dim=64, slots=67, recent=3, dtype=dt)
    m = Model(2, 4, 2, 64, 67, 3)
    for i in range(80):
        take_step(torch, cache, m, dt, 10 * i, f"step {i}")
    compare(torch, cache, m, "after 80 steps")


@pytest.mark.parametrize("H,Hk,K,d", [(4, 1, 5000, 128), (2, 2, 3001, 64), (24, 1, 2500, 128), (12, 1, 9000, 64), (16, 2, 1500, 128)])
def test_long_caches_cut_into_pieces(H, Hk, K, d):
    torch, P = _mods()
    for dt in types().values():
        cache, m = made(torch, P, 2, H, Hk, d, K, 40, dt, [K + 500, K // 3])
        for i in range(3):
            take_step(torch, cache, m, dt, 100 + 10 * i, f"{dt} step {i}")
        compare(torch, cache, m, str(dt))


def test_many_rows_with_two_thousand_slots():
    torch, P = _mods()
    dt = torch.bfloat16
    cache, m = made(torch, P, 4, 128, 128, 64, 2048, 40, dt, [2500, 2048, 2047, 10])
    for i in range(2):
        take_step(torch, cache, m, dt, 100 + 10 * i, f"step {i}")
    compare(torch, cache, m, "after")


def test_sharp_weights_and_another_scale():
    torch, P = _mods()
    for dt in types().values():
        cache, m = made(torch, P, 2, 4, 2, 128, 300, 10, dt, [400, 100], scale=0.5)
        for i in range(3):
            take_step(torch, cache, m, dt, 100 + 10 * i, f"{dt} step {i}", q_std=4.0)


def test_a_graph_replays_steps():
    torch, P = _mods()
    dt, shape = torch.bfloat16, dict(batch=3, heads=8, kv_heads=2, head_dim=128, slots=1200, recent=20, dtype=torch.bfloat16)
    k, v = draw(torch, (3, 2, 1500, 128), dt, 1), draw(torch, (3, 2, 1500, 128), dt, 2)
    scores = draw(torch, (3, 2, 1500), torch.float32, 3).abs()
    a, b = P.Q4Cache(**shape), P.Q4Cache(**shape)
    tokens = [[draw(torch, s, dt, 10 * i + j) for j, s in enumerate(((3, 8, 128), (3, 2, 128), (3, 2, 128)))] for i in range(4)]
    at = [x.clone() for x in tokens[0]]
    a.fill(k, v, scores)
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        a.step(*at)
    torch.cuda.current_stream().wait_stream(stream)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = a.step(*at)
    a.fill(k, v, scores)
    b.fill(k, v, scores)
    for i, x in enumerate(tokens):
        for to, y in zip(at, x):
            to.copy_(y)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, b.step(*x)), i
        for s, t in zip((a.cache, a.slot_pos, a.score, a.cursor), (b.cache, b.slot_pos, b.score, b.cursor)):
            assert torch.equal(s, t), i


def test_a_cursor_that_is_out_of_range_stays_within_its_row():
    """What a caller may hand over by mistake: the slot is cut off at the row's ends (the buffers around it stay as they are)."""
    torch, P = _mods()
    rows = torch.full((3, 1, 40), 7, dtype=torch.int32, device=DEV)
    for bad in (-5, 10 ** 6):
        cache = P.Q4Cache(batch=1, heads=1, kv_heads=1, head_dim=64, slots=40, recent=2, dtype=torch.bfloat16, slot_pos=rows[1:2].fill_(-1),
                          cursor=torch.tensor([[[bad, 3]]], dtype=torch.int32, device=DEV))
        x = draw(torch, (1, 1, 64), torch.bfloat16, 1)
        cache.step(x, x, x)
        torch.cuda.synchronize()
        assert bool((rows[0] == 7).all()) and bool((rows[2] == 7).all())
        slot = 0 if bad < 0 else 39
        assert int(cache.slot_pos[0, 0, slot]) == 3


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_what_free_slots_hold_does_not_matter(dtype):
    """Any bytes in the cache's free slots, scales of 0 and 255 among them (a buffer that nobody has cleared)."""
    torch, P = _mods()
    dt = types()[dtype]
    for H, K, byte in ((2, 100, 255), (2, 100, 0), (24, 70, 255), (8, 2000, 255)):
        cache = P.Q4Cache(batch=1, heads=H, kv_heads=1, head_dim=128, slots=K, recent=3, dtype=dt)
        cache.cache.fill_(byte)
        m = Model(1, H, 1, 128, K, 3)
        for i in range(3):
            take_step(torch, cache, m, dt, 10 * i, f"H {H} K {K} byte {byte} step {i}")
        compare(torch, cache, m, f"byte {byte}")
