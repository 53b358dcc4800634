"""GPU parity of attention over whole prompts (adore_prompt_attention, its gradients, adore_prompt_scores) against the definitions in
64 bits.

Tolerances, element by element, from the roundings there are.  A rounding to the storage type is off by at most half a unit,
u = eps / 2 of the value; fp32 sums of n products by at most n 2^-24 of the sum of their sizes (much less as a rule), so that a weight
p, whose exponent is such a sum, is off by t = 2^-24 (d max(scale |q|.|k|) + 8) of itself, and so is what is summed from weights.
  out     u |out| + (u + t) sum p |v|          (p is rounded where it enters the product)
  dv      u |dv| + (u + 2 t) sum p |do|
  dq      u |dq| + scale sum_j ((u + 2 t) |g| + (t + u_delta) p size) |k|, size = |do|.|v| + |do|.|out|
          u_delta: 2^-16 with what rounding out left (two roundings), u without, when u p |do|.(sum p |v|) |k| comes on top,
          from the weights that were rounded in out
  dk      the same over the queries and |q|
  lse     2^-24 (d max + 8 + |lse|) absolute;   scores  (2 t + 2^-20) of the score."""
import math

import numpy as np
import pytest

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TINY = 4096 * 2.0 ** -126      # weights below the smallest normal number of fp32 are zeros, up to 4096 of them in a sum


def _mods():
    import torch
    import paper_2407_02328_amd as P
    return torch, P


def reference(torch, q, k, v, do, scale):
    """One sequence, 64 bits: q, do [nq][H][d], k, v [nk][Hk][d].  Values and the sums that the bounds need."""
    q, k, v, do = (x.double() for x in (q, k, v, do))
    nq, H, d = q.shape
    nk, Hk, _ = k.shape
    g = H // Hk
    kh, vh = k.repeat_interleave(g, 1), v.repeat_interleave(g, 1)
    w = torch.einsum("ihd,jhd->hij", q, kh) * scale
    size = (torch.einsum("ihd,jhd->hij", q.abs(), kh.abs()) * scale).amax().item() if w.numel() else 0.0
    hidden = torch.ones((nq, nk), dtype=torch.bool, device=q.device).triu(nk - nq + 1)
    w = w.masked_fill(hidden, -math.inf)
    lse = torch.logsumexp(w, -1) if nk else torch.full((H, nq), -math.inf, dtype=torch.float64, device=q.device)
    p = torch.where(hidden, 0.0, torch.exp(w - lse[..., None]))
    p = torch.nan_to_num(p, nan=0.0)
    out = torch.einsum("hij,jhd->ihd", p, vh)
    r = dict(lse=lse, out=out, out_sum=torch.einsum("hij,jhd->ihd", p, vh.abs()), size=size)
    def group(x):
        return x.reshape(nk, Hk, g, d).sum(2)
    r["scores"] = p.sum(1).reshape(Hk, g, nk).sum(1)
    r["dv"], r["dv_sum"] = group(torch.einsum("hij,ihd->jhd", p, do)), group(torch.einsum("hij,ihd->jhd", p, do.abs()))
    dp = torch.einsum("ihd,jhd->hij", do, vh)
    delta = (do * out).sum(-1).t()
    far = torch.einsum("ihd,jhd->hij", do.abs(), vh.abs()) + (do.abs() * out.abs()).sum(-1).t()[..., None]
    gr = p * (dp - delta[..., None])
    r["dq"] = torch.einsum("hij,jhd->ihd", gr, kh) * scale
    r["dk"] = group(torch.einsum("hij,ihd->jhd", gr, q)) * scale
    out_far = (do.abs() * r["out_sum"]).sum(-1).t()[..., None]
    for name, x in (("g", gr.abs()), ("p", p * far), ("o", p * out_far)):
        r["dq_" + name] = torch.einsum("hij,jhd->ihd", x, kh.abs()) * scale
        r["dk_" + name] = group(torch.einsum("hij,ihd->jhd", x, q.abs())) * scale
    return r


def check(torch, got, want, dtype, d, rested=True, what=""):
    u = torch.finfo(dtype).eps / 2
    t = 2.0 ** -24 * (d * want["size"] + 8)
    ud = 0.0 if dtype == torch.float32 else 2.0 ** -16 if rested else u
    bound = {"out": u * want["out"].abs() + (u + t) * want["out_sum"]}
    bound["lse"] = 2.0 ** -24 * (d * want["size"] + 8 + want["lse"].abs())
    bound["scores"] = (2 * t + 2.0 ** -20) * want["scores"]
    bound["dv"] = u * want["dv"].abs() + (u + 2 * t) * want["dv_sum"]
    for x in ("dq", "dk"):
        bound[x] = u * want[x].abs() + (u + 2 * t) * want[x + "_g"] + (t + ud) * want[x + "_p"] + (0.0 if rested else u) * want[x + "_o"]
    for name, x in got.items():
        y = want[name]
        x = x.double()
        same = (x == y) | ((x - y).abs() <= bound[name] + TINY)
        assert bool(same.all()), f"{what} {name}: {int((~same).sum())} of {same.numel()} off, worst {((x - y).abs() - bound[name]).max().item()}"


def draw(torch, shape, dtype, seed, std=1.0):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return torch.empty(shape, dtype=dtype, device=DEV).normal_(0.0, std, generator=g)


def run_packed(torch, P, nq, nk, H, Hk, d, dtype, *, seed=1, std=1.0, scale=None, fused=False, rest=True, spare=3):
    """Packed sequences through all the entry points, with `spare` rows behind the last one; yields per sequence (got, want)."""
    Tq, Tk = sum(nq) + spare, sum(nk) + spare
    if fused:
        assert nq == nk
        qkv = draw(torch, (Tq, H + 2 * Hk, d), dtype, seed, std)
        q, k, v = qkv[:, :H], qkv[:, H:H + Hk], qkv[:, H + Hk:]
    else:
        q, k, v = draw(torch, (Tq, H, d), dtype, seed, std), draw(torch, (Tk, Hk, d), dtype, seed + 1, std), draw(torch, (Tk, Hk, d), dtype, seed + 2)
    do = draw(torch, (Tq, H, d), dtype, seed + 3)
    qs = torch.tensor(np.cumsum([0] + nq), dtype=torch.int32, device=DEV)
    ks = torch.tensor(np.cumsum([0] + nk), dtype=torch.int32, device=DEV)
    at = dict(q_start=qs, k_start=ks, scale=scale)
    out = torch.full((Tq, H, d), 7.0, dtype=dtype, device=DEV)
    out, lse, left = P.prompt_attention(q, k, v, out=out, rest=True, **at)
    grads = [torch.full(s, 7.0, dtype=dtype, device=DEV) for s in ((Tq, H, d), (Tk, Hk, d), (Tk, Hk, d))]
    dq, dk, dv = P.prompt_attention_backward(do, q, k, v, out, lse, rest=left if rest else None, dq=grads[0], dk=grads[1], dv=grads[2], **at)
    scores = P.prompt_scores(q, k, lse, scores=torch.full((Hk, Tk), 7.0, device=DEV), **at)
    torch.cuda.synchronize()
    if spare:
        for x in (out, dq, dk, dv, scores.t()):
            assert bool((x[-spare:] == 0.0).all()), "rows behind the last sequence are zeros"
        assert bool((lse[:, -spare:] == -math.inf).all())
    a = b = 0
    for n, m in zip(nq, nk):
        i, j = slice(a, a + n), slice(b, b + m)
        want = reference(torch, q[i], k[j], v[j], do[i], scale or d ** -0.5)
        yield dict(out=out[i], lse=lse[:, i], scores=scores[:, j], dq=dq[i], dk=dk[j], dv=dv[j]), want
        a, b = a + n, b + m


def bf16_f32():
    import torch
    return [torch.bfloat16, torch.float32]


LENGTHS = [
    ([1], [1]), ([1, 0, 2, 0, 33], [1, 0, 2, 0, 33]), ([31, 32, 33, 63, 64, 65], [31, 32, 33, 63, 64, 65]),
    ([127, 128, 129, 255, 257], [127, 128, 129, 255, 257]),
    ([1, 5, 64, 130], [200, 5, 65, 513]),              # a prefix that is there already
    ([40, 3, 130, 7], [10, 0, 129, 1]),                # first queries that see nothing, a sequence without keys
    ([0, 9], [17, 9]),                                 # a sequence without queries
]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("lengths", LENGTHS)
def test_packed_sequences(lengths, d, dtype):
    torch, P = _mods()
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    for H, Hk in ((2, 2), (6, 2)):
        for n, (got, want) in enumerate(run_packed(torch, P, *lengths, H, Hk, d, dt)):
            check(torch, got, want, dt, d, what=f"heads {H}/{Hk} sequence {n}")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("H,Hk,d", [(1, 1, 64), (3, 1, 128), (7, 7, 64), (16, 1, 64), (8, 8, 128), (24, 8, 64)])
def test_head_layouts(H, Hk, d, dtype):
    torch, P = _mods()
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    for n, (got, want) in enumerate(run_packed(torch, P, [70, 1, 300], [70, 1, 300], H, Hk, d, dt, fused=True)):
        check(torch, got, want, dt, d, what=f"sequence {n}")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_more_sequences_than_a_wave_has_lanes(dtype):
    torch, P = _mods()
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    rng = np.random.default_rng(5)
    lengths = [int(x) for x in rng.integers(0, 40, 150)]
    lengths[70] = 290
    for n, (got, want) in enumerate(run_packed(torch, P, lengths, lengths, 2, 1, 64, dt)):
        check(torch, got, want, dt, 64, what=f"sequence {n}")


@pytest.mark.parametrize("std,scale", [(8.0, None), (1.0, 1.0), (1e-4, None), (3.0, 0.01)])
def test_sharp_and_flat_weights(std, scale):
    torch, P = _mods()
    for dt in bf16_f32():
        for got, want in run_packed(torch, P, [333], [333], 2, 1, 128, dt, std=std, scale=scale):
            check(torch, got, want, dt, 128, what=str(dt))


def test_without_what_rounding_left():
    torch, P = _mods()
    for got, want in run_packed(torch, P, [5, 100], [5, 100], 4, 2, 64, torch.bfloat16, rest=False):
        check(torch, got, want, torch.bfloat16, 64, rested=False)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("B,H,Hk,nq,nk,d", [(2, 4, 2, 100, 100, 64), (1, 2, 2, 1, 1000, 128), (3, 2, 1, 129, 200, 128), (2, 3, 3, 64, 40, 64)])
def test_dense_batches(B, H, Hk, nq, nk, d, dtype):
    torch, P = _mods()
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    q, do = draw(torch, (B, H, nq, d), dt, 1), draw(torch, (B, nq, H, d), dt, 4).transpose(1, 2)     # another order of dimensions
    k, v = draw(torch, (B, Hk, nk, d), dt, 2), draw(torch, (B, Hk, nk, d), dt, 3)
    out, lse, rest = P.prompt_attention(q, k, v, rest=True)
    dq, dk, dv = P.prompt_attention_backward(do, q, k, v, out, lse, rest=rest)
    scores = P.prompt_scores(q, k, lse)
    for b in range(B):
        want = reference(torch, *(x[b].transpose(0, 1) for x in (q, k, v, do)), d ** -0.5)
        got = dict(out=out[b].transpose(0, 1), lse=lse[b], scores=scores[b], dq=dq[b].transpose(0, 1), dk=dk[b].transpose(0, 1), dv=dv[b].transpose(0, 1))
        check(torch, got, want, dt, d, what=f"sequence {b}")


def test_a_long_sequence():
    torch, P = _mods()
    dt, d = torch.bfloat16, 128
    for got, want in run_packed(torch, P, [2500], [3700], 3, 1, d, dt, spare=0):
        check(torch, got, want, dt, d)


def test_neighbours_that_are_not_numbers_do_not_reach_a_sequence():
    """NaN and infinities in the sequences before and behind, whose rows share tiles with it."""
    torch, P = _mods()
    for dt in bf16_f32():
        for bad in (math.nan, math.inf):
            q, k, v, do = (draw(torch, (140, 2, 64), dt, s) for s in (1, 2, 3, 4))
            for x in (q, k, v, do):
                x[:30] = bad
                x[107:] = bad
            at = dict(q_start=torch.tensor([0, 30, 107, 140], dtype=torch.int32, device=DEV), k_start=torch.tensor([0, 30, 107, 140], dtype=torch.int32, device=DEV))
            out, lse, rest = P.prompt_attention(q, k, v, rest=True, **at)
            dq, dk, dv = P.prompt_attention_backward(do, q, k, v, out, lse, rest=rest, **at)
            scores = P.prompt_scores(q, k, lse, **at)
            i = slice(30, 107)
            want = reference(torch, q[i], k[i], v[i], do[i], 64 ** -0.5)
            check(torch, dict(out=out[i], lse=lse[:, i], scores=scores[:, i], dq=dq[i], dk=dk[i], dv=dv[i]), want, dt, 64)


def test_gradients_against_differences():
    """sum(d_out . out) along a direction, by central differences of the forward pass in fp32: h = 2^-6 leaves h^2 / 6 of the third
    derivative (4e-5 of its size, at most some tens here) and 2 sqrt(n) 2^-24 / h of rounding."""
    torch, P = _mods()
    d, n = 64, 90
    q, k, v, do = (draw(torch, (n, h, d), torch.float32, s, 0.5) for h, s in ((4, 1), (2, 2), (2, 3), (4, 4)))
    at = dict(q_start=torch.tensor([0, 20, n], dtype=torch.int32, device=DEV), k_start=torch.tensor([0, 20, n], dtype=torch.int32, device=DEV))

    def loss(a, b, c):
        return float((P.prompt_attention(a, b, c, **at)[0].double() * do.double()).sum())

    out, lse = P.prompt_attention(q, k, v, **at)
    grads = P.prompt_attention_backward(do, q, k, v, out, lse, **at)
    h = 2.0 ** -6
    for n_, x in enumerate((q, k, v)):
        u = draw(torch, x.shape, torch.float32, 50 + n_)
        args = [q, k, v]
        hi, lo = list(args), list(args)
        hi[n_], lo[n_] = x + h * u, x - h * u
        slope = (loss(*hi) - loss(*lo)) / (2 * h)
        want = float((grads[n_].double() * u.double()).sum())
        size = float((grads[n_].double() * u.double()).square().sum().sqrt())       # of a sum of independent terms
        assert abs(slope - want) < 0.02 * size + 1e-3, (n_, slope, want, size)


def test_equal_inputs_give_equal_bits_and_a_graph_replays():
    torch, P = _mods()
    dt, d = torch.bfloat16, 128
    n = [300, 17, 129]
    T = sum(n)
    q, k, v, do = (draw(torch, (T, h, d), dt, s) for h, s in ((8, 1), (2, 2), (2, 3), (8, 4)))
    starts = torch.tensor(np.cumsum([0] + n), dtype=torch.int32, device=DEV)
    at = dict(q_start=starts, k_start=starts)

    def all_of_it():
        out, lse, rest = P.prompt_attention(q, k, v, rest=True, **at)
        return (out, lse, rest, *P.prompt_attention_backward(do, q, k, v, out, lse, rest=rest, **at), P.prompt_scores(q, k, lse, **at))

    want = [x.clone() for x in all_of_it()]
    for x, y in zip(all_of_it(), want):
        assert torch.equal(x, y)
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        all_of_it()
    torch.cuda.current_stream().wait_stream(stream)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = all_of_it()
    for turn in range(3):
        for x in got:
            x.fill_(3.0)
        q.mul_(1.0 if turn == 0 else 0.5)
        graph.replay()
        torch.cuda.synchronize()
        for x, y in zip(got, all_of_it()):
            assert torch.equal(x, y), turn


def test_scores_of_a_prompt_start_an_h2o_cache():
    """What the attention of a prompt gave its tokens, as adore_init_cache takes it: per (sequence, head) it adds up to the queries."""
    torch, P = _mods()
    q, k, v = (draw(torch, (2, 3, 77, 64), torch.bfloat16, s) for s in (1, 2, 3))
    out, lse = P.prompt_attention(q, k, v)
    scores = P.prompt_scores(q, k, lse)
    assert scores.shape == (2, 3, 77) and scores.is_contiguous()
    assert bool(((scores.double().sum(-1) - 77).abs() < 77 * 1e-5).all())
