"""Rotated heads, attention with a window, and the ring cache that serves it, as cases that can be measured.

Kinds of case (one pass of `run` each):

  rotate   rotate_heads: queries and keys of a projection, each head normed if the case has norms, turned by their tokens' positions
  turn     the same and its backward pass: gradients of q, k and the norms' weights
  attend   prompt_attention with a window: every query sees the last `window` keys up to its own and the first `sinks` ones
  train    the same and its backward pass: gradients of q, k and v
  fill     WindowCache.fill + read: the rows of prompts that the window and the first tokens leave, into the ring and out in order
  step     WindowCache.step: one token of every sequence through the ring: its row over the oldest one of the window, attention

`own` false: the operators in their plain form, elementary torch operations in 32 bits (angles in 64).  `own` true: the library's
calls.  Shapes are those of this repository's workloads and odder ones around them; all inputs are drawn on the device from the seed.

Rotation: pair j of the first `rotary` elements of a head, (j, j + rotary / 2) or, interleaved, (2 j, 2 j + 1), is turned by
position * f_j and stretched by `magnitude`; f_j = base^(-2 j / rotary), and with a factor those frequencies that make fewer than `low`
turns over the `original` length are divided by it, those that make more than `high` are not, in between the two are blended.

The ring: blocks of 32 slots, [K][V], each in the order in which the matrix instructions take its elements (_ring_of): position p is
in slot p if p < sinks, else in sinks + (p - sinks) % window.
"""
import math

import torch

own = False

DEV = "cuda"
BF16, F32 = "bf16", "f32"
TYPES = {BF16: torch.bfloat16, F32: torch.float32}
EPS = 1e-6


# ---- cases -----------------------------------------------------------------------------------------------------


def _rotate(name, kind, *, batch, tokens, heads, kv, d, rotary, interleaved=False, norm=False, base=10000.0, factor=1.0, original=4096,
            past=0, dtype=BF16):
    """Packed sequences of 1 to `tokens` tokens (_lengths; all of one token if that is 1), each behind up to `past` others."""
    case = dict(kind=kind, batch=batch, tokens=tokens, heads=heads, kv=kv, d=d, rotary=rotary, interleaved=interleaved, norm=norm, base=base,
                factor=factor, original=original, past=past, dtype=dtype)
    return dict(case, name=name) if name else case


def _prompt(name, kind, *, batch, tokens, heads, kv, d, window, sinks, past=0, ragged=True, dtype=BF16):
    """ragged: packed sequences of 1 to `tokens` tokens (_lengths); else a dense batch of `tokens` tokens each, [B][H][S][d].
    past: keys of every sequence that are there before its first query (a prompt taken in by pieces)."""
    case = dict(kind=kind, batch=batch, tokens=tokens, heads=heads, kv=kv, d=d, window=window, sinks=sinks, past=past, ragged=ragged, dtype=dtype)
    return dict(case, name=name) if name else case


def _ring(name, kind, *, batch, heads, kv, d, window, sinks, tokens, dtype=BF16):
    """tokens: that the longest sequence has had (_lengths: the others fewer; of a fill's packed prompts, and of a step's cache)."""
    case = dict(kind=kind, batch=batch, heads=heads, kv=kv, d=d, window=window, sinks=sinks, tokens=tokens, dtype=dtype)
    return dict(case, name=name) if name else case


def listed():
    return [
        # one token of the ordinary serving batch, on its way into a cache
        _rotate("rotate_token", "rotate", batch=16, tokens=1, heads=32, kv=32, d=128, rotary=128, past=1024),
        # the prompts of many requests of a 7B-shaped layer, of very different lengths
        _rotate("rotate_packed_prompts", "rotate", batch=40, tokens=1024, heads=32, kv=32, d=128, rotary=128),
        # fine-tuning a small fp32 model for longer texts than it knows: half of the head, pairs side by side, frequencies scaled
        _rotate("turn_small_f32", "turn", batch=7, tokens=333, heads=12, kv=4, d=64, rotary=32, interleaved=True, factor=8.0, past=30000, dtype=F32),
        # fine-tuning a 7B-shaped layer with grouped heads and norms of queries and keys
        _rotate("turn_normed_grouped", "turn", batch=40, tokens=2048, heads=32, kv=8, d=128, rotary=128, norm=True, base=500000.0),
        # long documents under a window
        _prompt("attend_long_window", "attend", batch=2, tokens=8192, heads=32, kv=4, d=128, window=1020, sinks=4, ragged=False),
        # requests of very different lengths in one launch, grouped heads, an odd window, no first tokens
        _prompt("attend_packed_window", "attend", batch=24, tokens=2777, heads=32, kv=8, d=64, window=501, sinks=0),
        # a few short packed texts of a small fp32 model: latency
        _prompt("train_tiny_window_f32", "train", batch=3, tokens=128, heads=4, kv=4, d=64, window=32, sinks=4, dtype=F32),
        # fine-tuning a 7B-shaped layer with grouped heads under the window that it is to be served with
        _prompt("train_grouped_window", "train", batch=8, tokens=2048, heads=32, kv=8, d=128, window=508, sinks=4, ragged=False),
        # prompts of all lengths into the rings that their answers are made with: the ordinary batch, and a few odd ones in fp32
        _ring("fill_llama7b_layer", "fill", batch=16, heads=32, kv=32, d=128, window=508, sinks=4, tokens=1024),
        _ring("fill_odd_f32", "fill", batch=5, heads=12, kv=12, d=64, window=200, sinks=3, tokens=777, dtype=F32),
        # one token of the ordinary batch: most rings are full, some are not
        _ring("step_llama7b_layer", "step", batch=16, heads=32, kv=32, d=128, window=508, sinks=4, tokens=4096),
        # a few sequences with long windows and grouped heads
        _ring("step_long_grouped", "step", batch=4, heads=32, kv=8, d=128, window=16380, sinks=4, tokens=100000),
    ]


def _log_int(rng, lo, hi):
    return min(hi, int(math.exp(rng.uniform(math.log(lo), math.log(hi + 1)))))


def draw(rng):
    kind = rng.choice(["rotate", "turn", "attend", "attend", "train", "train", "fill", "step", "step"])
    while True:
        d = rng.choice([64, 128])
        kv = rng.choice([1, 2, 4, 8, 12, 32])
        heads = kv * rng.choice([g for g in (1, 2, 3, 4, 7, 8, 16) if kv * g <= 64])
        dtype = F32 if rng.random() < 0.25 else BF16
        sinks = rng.choice([0, 1, 4, rng.randint(0, 64)])
        if kind in ("rotate", "turn"):
            batch, tokens = _log_int(rng, 1, 64), rng.choice([1, _log_int(rng, 1, 4096)])
            if batch * tokens * (heads + kv) * d <= 1 << 27:
                return _rotate(None, kind, batch=batch, tokens=tokens, heads=heads, kv=kv, d=d, rotary=rng.choice([d, d, d // 2, 16, 3 * d // 4]),
                               interleaved=rng.random() < 0.4, norm=rng.random() < 0.5, base=rng.choice([10000.0, 500000.0]),
                               factor=rng.choice([1.0, 1.0, 4.0, 32.0]), past=rng.choice([0, _log_int(rng, 1, 1 << 20)]), dtype=dtype)
        elif kind in ("attend", "train"):
            batch, tokens = _log_int(rng, 1, 32), _log_int(rng, 48, 8192)
            past = _log_int(rng, 1, 4096) if rng.random() < 0.25 else 0
            padded = batch * heads * tokens * (tokens + past)
            if padded <= (1 << 28 if dtype == F32 else 1 << 30 if kind == "train" else 1 << 31) and batch * (tokens + past) * heads >= 2048:
                return _prompt(None, kind, batch=batch, tokens=tokens, heads=heads, kv=kv, d=d, window=_log_int(rng, 2, tokens), sinks=sinks,
                               past=past, ragged=rng.random() < 0.7, dtype=dtype)
        else:
            batch, window = _log_int(rng, 1, 64), _log_int(rng, 16, 16384)
            tokens = _log_int(rng, max(1, window // 4), 4 * window)
            if kind == "fill" and batch * kv * max(tokens, window + sinks) * d <= 1 << 26 or kind == "step" and 256 <= batch * kv * window <= 1 << 19:
                return _ring(None, kind, batch=batch, heads=heads, kv=kv, d=d, window=window, sinks=sinks, tokens=tokens, dtype=dtype)


def _lengths(batch, longest):
    """The longest first, then others spread over 1 .. longest, many short ones (squares of an even spread)."""
    return [longest if i == 0 else max(1, round(longest * math.modf(0.3 + 0.618033988749895 * i)[0] ** 2)) for i in range(batch)]


def _q_lengths(c):
    return _lengths(c["batch"], c["tokens"]) if c.get("ragged", True) else [c["tokens"]] * c["batch"]


# ---- inputs ----------------------------------------------------------------------------------------------------


class _Draws:
    def __init__(self, seed):
        self.g = torch.Generator(device=DEV)
        self.g.manual_seed(seed)

    def normal(self, shape, dtype):
        return torch.empty(shape, dtype=dtype, device=DEV).normal_(0.0, 1.0, generator=self.g)


class _State:
    def __init__(self, case):
        self.case = case
        self.handle = None


def _starts(lengths):
    return torch.tensor([0] + torch.tensor(lengths).cumsum(0).tolist(), dtype=torch.int32, device=DEV)


def _prepare_rotate(c, seed):
    r, s = _Draws(seed), _State(c)
    st, Hq, Hk, d = TYPES[c["dtype"]], c["heads"], c["kv"], c["d"]
    n = _q_lengths(c)
    behind = [p if c["past"] else 0 for p in reversed(_lengths(c["batch"], max(1, c["past"])))]
    s.positions = torch.cat([torch.arange(p, p + m, dtype=torch.int32, device=DEV) for m, p in zip(n, behind)])
    qkv = r.normal((sum(n), Hq + 2 * Hk, d), st)   # as the projection of all three leaves them
    s.q, s.k = qkv[:, :Hq], qkv[:, Hq:Hq + Hk]
    s.q_weight = s.k_weight = None
    if c["norm"]:
        s.q_weight, s.k_weight = (1.0 + 0.2 * r.normal((d,), torch.float32) for _ in range(2))
    if c["kind"] == "turn":
        s.d_q, s.d_k = r.normal(tuple(s.q.shape), st), r.normal(tuple(s.k.shape), st)
    return s


def _prepare_prompt(c, seed):
    r, s = _Draws(seed), _State(c)
    st, B, Hq, Hk, d = TYPES[c["dtype"]], c["batch"], c["heads"], c["kv"], c["d"]
    nq = _q_lengths(c)
    nk = [n + c["past"] for n in nq]
    s.q_start = s.k_start = None
    if c["ragged"]:
        s.q_start, s.k_start = _starts(nq), _starts(nk)
        Tq, Tk = sum(nq), sum(nk)
        if c["past"]:
            s.q, s.k, s.v = r.normal((Tq, Hq, d), st), r.normal((Tk, Hk, d), st), r.normal((Tk, Hk, d), st)
        else:                                      # as the projection of all three leaves them
            qkv = r.normal((Tq, Hq + 2 * Hk, d), st)
            s.q, s.k, s.v = qkv[:, :Hq], qkv[:, Hq:Hq + Hk], qkv[:, Hq + Hk:]
    else:
        s.q, s.k, s.v = r.normal((B, Hq, nq[0], d), st), r.normal((B, Hk, nk[0], d), st), r.normal((B, Hk, nk[0], d), st)
    if c["kind"] == "train":
        s.d_out = r.normal(tuple(s.q.shape), st)
    return s


def _ring_of(k, v):
    """K and V [B][H][32 n][d] to the ring's elements [B][H][n][64 d]."""
    if k.dtype == torch.float32:
        kb = k.unflatten(3, (-1, 4, 4)).unflatten(2, (-1, 2, 16)).permute(0, 1, 2, 5, 3, 6, 4, 7)      # b h n | t c | s q i -> s t q c i
        vb = v.unflatten(3, (-1, 16)).unflatten(2, (-1, 2, 4, 4)).permute(0, 1, 2, 6, 3, 4, 7, 5)      # b h n | t q i | s c -> s t q c i
    else:
        kb = k.unflatten(3, (-1, 4, 8)).unflatten(2, (-1, 4, 2, 4)).permute(0, 1, 2, 6, 4, 7, 3, 5, 8)  # b h n | a t e | s q i -> s t q a e i
        vb = v.unflatten(3, (-1, 16)).unflatten(2, (-1, 4, 8)).permute(0, 1, 2, 5, 3, 6, 4)             # b h n | q i | s c -> s q c i
    return torch.cat([kb.flatten(3), vb.flatten(3)], -1).contiguous()


def _rows_of(ring, d):
    """Inverse of _ring_of."""
    kb, vb = ring.split(32 * d, -1)
    if ring.dtype == torch.float32:
        k = kb.unflatten(3, (d // 16, 2, 4, 16, 4)).permute(0, 1, 2, 4, 6, 3, 5, 7)
        v = vb.unflatten(3, (d // 16, 2, 4, 16, 4)).permute(0, 1, 2, 4, 5, 7, 3, 6)
    else:
        k = kb.unflatten(3, (d // 32, 2, 4, 4, 4, 8)).permute(0, 1, 2, 6, 4, 7, 3, 5, 8)
        v = vb.unflatten(3, (d // 16, 4, 16, 8)).permute(0, 1, 2, 4, 6, 3, 5)
    shape = (ring.shape[0], ring.shape[1], 32 * ring.shape[2], d)
    return k.reshape(shape), v.reshape(shape)


def _held_positions(c, tokens):
    """Positions in slot order [B][slots] of sequences that have had `tokens` [B], -1 in free slots."""
    W, S = c["window"], c["sinks"]
    slot, n = torch.arange(W + S, device=DEV), tokens[:, None].long()
    behind = (n - 1 - slot).clamp(min=0) // W * W        # (the window's slots: the last position that is in the slot)
    pos = torch.where(slot < S, slot, slot + behind)
    return torch.where(slot < n, pos, -1)


def _prepare_ring(c, seed):
    r, s = _Draws(seed), _State(c)
    st, B, Hq, H, d = TYPES[c["dtype"]], c["batch"], c["heads"], c["kv"], c["d"]
    slots = c["window"] + c["sinks"]
    n = _lengths(B, c["tokens"])
    shape = (B, H, (slots + 31) // 32, 64 * d)
    if c["kind"] == "fill":
        s.k_start = _starts(n)
        s.k, s.v = r.normal((sum(n), H, d), st), r.normal((sum(n), H, d), st)
        s.ring = torch.zeros(shape, dtype=st, device=DEV)
        s.cursor = torch.zeros((B, H), dtype=torch.int32, device=DEV)
    else:
        s.cursor = torch.tensor(n, dtype=torch.int32, device=DEV)[:, None].expand(B, H).contiguous()
        s.ring = r.normal(shape, st)                # (any order of normal elements is one: free slots hold some too)
        s.q, s.k, s.v = r.normal((B, Hq, d), st), r.normal((B, H, d), st), r.normal((B, H, d), st)
    return s


def prepare(case, seed):
    kind = case["kind"]
    return (_prepare_rotate if kind in ("rotate", "turn") else _prepare_prompt if kind in ("attend", "train") else _prepare_ring)(case, seed)


# ---- plain forms -------------------------------------------------------------------------------------------------


def _magnitude(c):
    return 0.1 * math.log(c["factor"]) + 1.0


def _frequencies(c):
    """Of the pairs, in 64 bits."""
    f = c["base"] ** (-2.0 * torch.arange(c["rotary"] // 2, dtype=torch.float64, device=DEV) / c["rotary"])
    if c["factor"] == 1.0:
        return f
    whole = ((c["original"] * f / (2.0 * math.pi) - 1.0) / 31.0).clamp(0.0, 1.0)      # from 1 turn to 32
    return f * (whole + (1.0 - whole) / c["factor"])


def _pairs(x, c):
    """The two elements of every pair, and what is not turned."""
    R = c["rotary"]
    a, b = (x[..., 0:R:2], x[..., 1:R:2]) if c["interleaved"] else (x[..., :R // 2], x[..., R // 2:R])
    return a, b, x[..., R:]


def _joined(a, b, rest, c):
    turned = torch.stack([a, b], -1).flatten(-2) if c["interleaved"] else torch.cat([a, b], -1)
    return torch.cat([turned, rest], -1)


def _plain_rotate(s):
    c, st = s.case, s.q.dtype
    t = s.positions.double()[:, None] * _frequencies(c)
    cos, sin = ((_magnitude(c) * f(t)).float()[:, None] for f in (torch.cos, torch.sin))

    def forward(x, weight):
        y = x.float()
        if weight is not None:
            y = y * torch.rsqrt(y.square().mean(-1, keepdim=True) + EPS) * weight
        a, b, rest = _pairs(y, c)
        return _joined(a * cos - b * sin, a * sin + b * cos, rest, c).to(st)

    def backward(d_out, x, weight):
        a, b, rest = _pairs(d_out.float(), c)
        g = _joined(a * cos + b * sin, b * cos - a * sin, rest, c)
        if weight is None:
            return g.to(st), None
        x = x.float()
        r = torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS)
        n, wg = x * r, g * weight
        return (r * (wg - n * (wg * n).mean(-1, keepdim=True))).to(st), (g * n).double().sum((0, 1)).float()

    result = {"q": forward(s.q, s.q_weight), "k": forward(s.k, s.k_weight)}
    if c["kind"] == "turn":
        result["dq"], dqw = backward(s.d_q, s.q, s.q_weight)
        result["dk"], dkw = backward(s.d_k, s.k, s.k_weight)
        if c["norm"]:
            result.update(dq_weight=dqw, dk_weight=dkw)
    return result


def _places(start, batch, longest):
    """Row of token t of sequence b (row 0 where there is none), [B][longest], and which are there."""
    t = torch.arange(longest, device=DEV)
    there = t < (start[1:] - start[:-1])[:, None]
    return torch.where(there, start[:-1, None] + t, 0).long(), there


def _padded(s):
    """q [B][Hk][g][Sq][d], k, v [B][Hk][Sk][d] in 32 bits, which keys a query sees [B][1][1][Sq][Sk], and where rows belong."""
    c = s.case
    B, Hq, Hk, Sq = c["batch"], c["heads"], c["kv"], c["tokens"]
    Sk = Sq + c["past"]
    j, p = torch.arange(Sk, device=DEV), torch.arange(Sq, device=DEV)[:, None] + c["past"]
    q, k, v, where = s.q, s.k, s.v, (None, None)
    seen = ((j <= p) & ((p - j < c["window"]) | (j < c["sinks"]))).expand(B, Sq, Sk)
    if c["ragged"]:
        at_q, there_q = _places(s.q_start, B, Sq)
        at_k, there_k = _places(s.k_start, B, Sk)
        q, k, v = (x[at].transpose(1, 2) for x, at in ((q, at_q), (k, at_k), (v, at_k)))
        seen = seen & there_q[:, :, None] & there_k[:, None, :]
        where = (there_q, there_k)
    return q.float().unflatten(1, (Hk, Hq // Hk)), k.float(), v.float(), seen[:, None, None], where


def _rows(x, there):
    """[B][H][S][d] to the packed [T][H][d] (or as it is)."""
    return x.contiguous() if there is None else x.transpose(1, 2)[there]


def _row_values(x, there):
    """[B][H..][S] to the packed [H][T] (or [B][H][S])."""
    x = x.flatten(1, 2)
    return x.contiguous() if there is None else x.transpose(1, 2)[there].t().contiguous()


def _plain_attend(s, backward):
    c, st = s.case, s.q.dtype
    scale = c["d"] ** -0.5
    q, k, v, seen, where = _padded(s)
    w = (q.flatten(2, 3) @ k.transpose(-1, -2).contiguous()).mul_(scale).unflatten(2, q.shape[2:4]).masked_fill_(~seen, -math.inf)
    top = w.amax(-1, keepdim=True).clamp_(min=-1e30)
    p = w.sub_(top).exp_()
    l = p.sum(-1, keepdim=True)
    lse = (top + l.log())[..., 0]
    p /= torch.where(l > 0, l, 1.0)
    out = (p.flatten(2, 3) @ v).unflatten(2, q.shape[2:4])
    result = {"out": _rows(out.flatten(1, 2), where[0]).to(st), "lse": _row_values(lse, where[0])}
    if not backward:
        return result
    do = s.d_out if where[0] is None else s.d_out[_places(s.q_start, c["batch"], c["tokens"])[0]].transpose(1, 2)
    do = do.float().unflatten(1, q.shape[1:3])
    do = do if where[0] is None else torch.where(where[0][:, None, None, :, None], do, 0.0)
    flat = do.flatten(2, 3)
    dv = p.flatten(2, 3).transpose(-1, -2).contiguous() @ flat
    dp = (flat @ v.transpose(-1, -2).contiguous()).unflatten(2, q.shape[2:4])
    ds = dp.sub_((p * dp).sum(-1, keepdim=True)).mul_(p).mul_(scale).flatten(2, 3)
    dq = (ds @ k).unflatten(2, q.shape[2:4]).flatten(1, 2)
    dk = ds.transpose(-1, -2).contiguous() @ q.flatten(2, 3)
    return dict(result, dq=_rows(dq, where[0]).to(st), dk=_rows(dk, where[1]).to(st), dv=_rows(dv, where[1]).to(st))


def _plain_fill(s):
    c = s.case
    W, S, d = c["window"], c["sinks"], c["d"]
    tokens = (s.k_start[1:] - s.k_start[:-1]).long()
    pos = _held_positions(c, tokens)                                   # [B][slots]
    at = s.k_start[:-1, None].long() + pos.clamp(min=0)
    more = -(W + S) % 32

    def held(x):
        rows = torch.where((pos >= 0)[..., None, None], x[at], 0.0).transpose(1, 2)
        return torch.nn.functional.pad(rows, (0, 0, 0, more))

    s.ring.copy_(_ring_of(held(s.k), held(s.v)))
    s.cursor.copy_(tokens[:, None].expand(s.cursor.shape))
    # out in the order of positions: free slots last
    order = torch.where(pos >= 0, pos, 1 << 40).argsort(-1)[:, None, :, None].expand(-1, c["kv"], -1, d)
    k, v = (x[:, :, :W + S].gather(2, order) for x in _rows_of(s.ring, d))
    return {"k": k, "v": v, "cursor": s.cursor}


def _plain_step(s):
    c, st = s.case, s.q.dtype
    W, S, d, H = c["window"], c["sinks"], c["d"], c["kv"]
    n = s.cursor[:, 0].long()
    slot = torch.where(n < S, n, S + (n - S) % W)
    k, v = _rows_of(s.ring, d)
    at = slot[:, None, None, None].expand(-1, H, 1, d)
    k, v = k.scatter(2, at, s.k[:, :, None]), v.scatter(2, at, s.v[:, :, None])
    s.ring.copy_(_ring_of(k, v))
    there = torch.arange(k.shape[2], device=DEV) < (n + 1).clamp(max=W + S)[:, None]
    w = (s.q.float().unflatten(1, (H, -1)) @ k.float().transpose(-1, -2).contiguous()) * d ** -0.5
    w = w.masked_fill(~there[:, None, None], -math.inf)
    p = (w - w.amax(-1, keepdim=True)).exp()
    p = p / p.sum(-1, keepdim=True)
    out = p @ torch.where(there[:, None, :, None], v.float(), 0.0)
    s.cursor += 1
    return {"out": out.flatten(1, 2).to(st), "ring": s.ring, "cursor": s.cursor}


# ---- one pass ----------------------------------------------------------------------------------------------------


def _handle(s):
    """The rotation or the ring as a user's program keeps it: made once."""
    if s.handle is None:
        from paper_2407_02328_amd import Rotary, WindowCache
        c = s.case
        if c["kind"] in ("rotate", "turn"):
            scaled = {} if c["factor"] == 1.0 else dict(factor=c["factor"], original=c["original"], low=1.0, high=32.0, magnitude=_magnitude(c))
            s.handle = Rotary(c["rotary"], base=c["base"], interleaved=c["interleaved"], **scaled)
        else:
            s.handle = WindowCache(batch=c["batch"], heads=c["heads"], kv_heads=c["kv"], head_dim=c["d"], window=c["window"], sinks=c["sinks"],
                                   dtype=c["dtype"], cache=s.ring, cursor=s.cursor)
    return s.handle


def _own_rotate(s):
    from paper_2407_02328_amd import rotate_heads, rotate_heads_backward
    h, c = _handle(s), s.case
    norms = dict(q_weight=s.q_weight, k_weight=s.k_weight, eps=EPS)
    q, k = rotate_heads(s.q, s.k, s.positions, h, **norms)
    if c["kind"] == "rotate":
        return {"q": q, "k": k}
    dq, dk, dqw, dkw = rotate_heads_backward(s.d_q, s.d_k, s.q, s.k, s.positions, h, **norms)
    result = {"q": q, "k": k, "dq": dq, "dk": dk}
    return dict(result, dq_weight=dqw, dk_weight=dkw) if c["norm"] else result


def _own_attend(s):
    from paper_2407_02328_amd import prompt_attention, prompt_attention_backward
    c = s.case
    how = dict(q_start=s.q_start, k_start=s.k_start, window=c["window"], sinks=c["sinks"])
    if c["kind"] == "attend":
        out, lse = prompt_attention(s.q, s.k, s.v, **how)
        return {"out": out, "lse": lse}
    out, lse, rest = prompt_attention(s.q, s.k, s.v, rest=True, **how)
    dq, dk, dv = prompt_attention_backward(s.d_out, s.q, s.k, s.v, out, lse, rest=rest, **how)
    return {"out": out, "lse": lse, "dq": dq, "dk": dk, "dv": dv}


def _own_ring(s):
    h = _handle(s)
    if s.case["kind"] == "fill":
        h.fill(s.k, s.v, k_start=s.k_start)
        k, v = h.read()
        return {"k": k, "v": v, "cursor": s.cursor}
    return {"out": h.step(s.q, s.k, s.v), "ring": s.ring, "cursor": s.cursor}


def run(s):
    kind = s.case["kind"]
    if kind in ("rotate", "turn"):
        return _own_rotate(s) if own else _plain_rotate(s)
    if kind in ("attend", "train"):
        return _own_attend(s) if own else _plain_attend(s, kind == "train")
    return _own_ring(s) if own else _plain_fill(s) if kind == "fill" else _plain_step(s)


# ---- what a pass cannot do without -------------------------------------------------------------------------------


def work(case):
    c = case
    es, d, Hq, H = 2 if c["dtype"] == BF16 else 4, c["d"], c["heads"], c["kv"]
    n = _lengths(c["batch"], c["tokens"])
    if c["kind"] in ("rotate", "turn"):
        rows = float(sum(n) * (Hq + H) * d * es)
        # q, k in and out, positions; the backward pass: gradients in and out, q and k once more where norms want them
        passes = 2 if c["kind"] == "rotate" else 5 if c["norm"] else 4
        return {"bytes": passes * rows + 4.0 * sum(n), "flops": 3.0 * (passes - 1) * rows / es}
    if c["kind"] in ("attend", "train"):
        nq, past, W, S = _q_lengths(c), c["past"], c["window"], c["sinks"]
        Tq, Tk = sum(nq), sum(nq) + past * c["batch"]

        def upto(m, most):                         # the sum of min(t, most) over t = 1 .. m
            full = min(m, most)
            return full * (full + 1) // 2 + max(0, m - most) * most

        # token t (from 1) sees min(t, W) keys of its window and min(max(t - W, 0), S) first ones before it
        pairs = Hq * sum(upto(m + past, W) - upto(past, W) + upto(max(0, m + past - W), S) - upto(max(0, past - W), S) for m in nq)
        q, k, rows = Tq * Hq * d * es, Tk * H * d * es, 4.0 * Tq * Hq
        if c["kind"] == "attend":
            return {"bytes": 2.0 * q + 2.0 * k + rows, "flops": 4.0 * d * pairs}
        return {"bytes": 4.0 * q + 4.0 * k + rows, "flops": 14.0 * d * pairs}      # q, k, v, d_out in; out and three gradients out
    slots = c["window"] + c["sinks"]
    if c["kind"] == "fill":
        kept = H * sum(min(x, slots) for x in n) * d * es
        # kept rows in, to the ring, and back; the contents out
        return {"bytes": 6.0 * kept + 2.0 * H * c["batch"] * slots * d * es, "flops": 0.0}
    held = H * sum(min(x + 1, slots) for x in n)
    return {"bytes": 2.0 * held * d * es + c["batch"] * (2 * Hq + 2 * H) * d * es, "flops": 4.0 * d * held * (Hq // H)}


# ---- from the definitions, in 64 bits ------------------------------------------------------------------------------


def _exact_rotate(s):
    c, d = s.case, s.case["d"]
    R = c["rotary"]
    # the whole rotation of a token as a complex number for each pair, by its definition
    f = torch.tensor([c["base"] ** (-2.0 * j / R) for j in range(R // 2)], dtype=torch.float64, device=DEV)
    if c["factor"] != 1.0:
        turns = c["original"] * f / (2.0 * math.pi)
        share = torch.where(turns <= 1.0, 0.0, torch.where(turns >= 32.0, 1.0, (turns - 1.0) / 31.0))
        f = f / c["factor"] * (1.0 - share) + f * share
    z = torch.polar(torch.full((1,), 1.0 if c["factor"] == 1.0 else 1.0 + math.log(c["factor"]) / 10.0, dtype=torch.float64, device=DEV),
                    s.positions.double()[:, None] * f)[:, None]
    if c["interleaved"]:
        first = torch.arange(0, R, 2, device=DEV)
        second = first + 1
    else:
        first = torch.arange(R // 2, device=DEV)
        second = first + R // 2

    def turned(x, by):
        w = torch.complex(x[..., first], x[..., second]) * by
        y = x.clone()
        y[..., first], y[..., second] = w.real, w.imag
        return y

    def normed(x, weight):
        return x if weight is None else x / torch.sqrt((x * x).sum(-1, keepdim=True) / d + EPS) * weight.double()

    res = {"q": turned(normed(s.q.double(), s.q_weight), z), "k": turned(normed(s.k.double(), s.k_weight), z)}
    if c["kind"] == "turn":
        for name, d_out, x, weight in (("q", s.d_q, s.q.double(), s.q_weight), ("k", s.d_k, s.k.double(), s.k_weight)):
            g = turned(d_out.double(), z.conj())
            if weight is not None:
                size = torch.sqrt((x * x).sum(-1, keepdim=True) / d + EPS)
                res["d" + name + "_weight"] = (g * x / size).flatten(0, 1).sum(0)
                g = g * weight.double()
                g = g / size - x * ((g * x).sum(-1, keepdim=True) / (d * size ** 3))
            res["d" + name] = g
    return res


def _exact_prompt(s):
    c, ragged = s.case, s.case["ragged"]
    d, g, past = c["d"], c["heads"] // c["kv"], c["past"]
    f = dict(dtype=torch.float64, device=DEV)
    res = {"out": torch.zeros(s.q.shape, **f), "lse": torch.zeros((c["heads"], s.q.shape[0]) if ragged else s.q.shape[:3], **f)}
    if c["kind"] == "train":
        res.update(dq=torch.zeros(s.q.shape, **f), dk=torch.zeros(s.k.shape, **f), dv=torch.zeros(s.v.shape, **f))
    a = e = 0
    for b, n in enumerate(_q_lengths(c)):
        m = n + past
        visible = torch.ones((n, m), dtype=torch.bool, device=DEV).tril(past)
        outside = torch.ones((n, m), dtype=torch.bool, device=DEV).tril(past - c["window"])
        outside[:, :c["sinks"]] = False
        hidden = outside | ~visible
        for h in range(c["heads"]):
            def of(x, first, count, head):
                return (x[first:first + count, head] if ragged else x[b, head])

            q, k, v = (of(x, *at).double() for x, at in ((s.q, (a, n, h)), (s.k, (e, m, h // g)), (s.v, (e, m, h // g))))
            w = torch.exp(q @ k.t() / math.sqrt(d))
            w[hidden] = 0.0
            total = w.sum(1)
            p = w / total[:, None]
            o = p @ v
            of(res["out"], a, n, h).add_(o)
            (res["lse"][h, a:a + n] if ragged else res["lse"][b, h]).add_(total.log())
            if c["kind"] == "train":
                do = of(s.d_out, a, n, h).double()
                of(res["dv"], e, m, h // g).add_(p.t() @ do)
                ds = p * (do @ v.t() - (do * o).sum(1, keepdim=True)) / math.sqrt(d)
                of(res["dq"], a, n, h).add_(ds @ k)
                of(res["dk"], e, m, h // g).add_(ds.t() @ q)
        a, e = a + n, e + m
    return res


def _exact_fill(s):
    c = s.case
    B, H, d, W, S = c["batch"], c["kv"], c["d"], c["window"], c["sinks"]
    k, v = (torch.zeros((B, H, W + S, d), dtype=torch.float64, device=DEV) for _ in range(2))
    first = 0
    for b, n in enumerate(_lengths(B, c["tokens"])):
        for to, x in ((k, s.k), (v, s.v)):
            rows = x[first:first + n].double().transpose(0, 1)
            kept = rows if n <= W + S else torch.cat([rows[:, :S], rows[:, n - W:]], 1)
            to[b, :, :kept.shape[1]] = kept
        first += n
    return {"k": k, "v": v, "cursor": None}


def _exact_step(s):
    c = s.case
    B, H, d, W, S = c["batch"], c["kv"], c["d"], c["window"], c["sinks"]
    g, slots = c["heads"] // H, W + S
    n = s.cursor[:, 0].tolist()
    # where element e of slot x is within its block
    x, e = torch.arange((slots + 31) // 32 * 32, device=DEV)[:, None], torch.arange(d, device=DEV)
    i, block = x % 32, x // 32 * (64 * d)
    if s.q.dtype == torch.float32:
        at_k = block + (e // 16 * 2 + i // 16) * 256 + e // 4 % 4 * 64 + i % 16 * 4 + e % 4
        at_v = block + 32 * d + (e // 16 * 2 + i // 16) * 256 + i // 4 % 4 * 64 + e % 16 * 4 + i % 4
    else:
        at_k = block + (e // 32 * 2 + i // 4 % 2) * 512 + e // 8 % 4 * 128 + (i // 8 * 4 + i % 4) * 8 + e % 8
        at_v = block + 32 * d + e // 16 * 512 + i // 8 * 128 + e % 16 * 8 + i % 8
    ring = s.ring.flatten(2).double()
    out = torch.zeros((B, c["heads"], d), dtype=torch.float64, device=DEV)
    for b in range(B):
        at = n[b] if n[b] < S else S + (n[b] - S) % W
        ring[b][:, at_k[at]], ring[b][:, at_v[at]] = s.k[b].double(), s.v[b].double()
        held = min(n[b] + 1, slots)
        for h in range(H):
            kk, vv = ring[b, h][at_k[:held]], ring[b, h][at_v[:held]]
            p = torch.softmax(s.q[b, h * g:(h + 1) * g].double() @ kk.t() / math.sqrt(d), -1)
            out[b, h * g:(h + 1) * g] = p @ vv
    return {"out": out, "ring": ring.view(s.ring.shape), "cursor": None}


def exact(case, seed):
    s = prepare(case, seed)
    kind = case["kind"]
    if kind in ("rotate", "turn"):
        return _exact_rotate(s)
    return _exact_prompt(s) if kind in ("attend", "train") else _exact_fill(s) if kind == "fill" else _exact_step(s)
