"""GPU parity of attention with a window and first tokens that stay visible (adore_window_attention and its gradients) against the
definitions in 64 bits: the query at position p sees keys j <= p with p - j < window or j < sinks.

Tolerances as in test_gpu_prompt.py, whose derivation knows nothing of which keys are seen: weights rounded to the storage type where
they enter a product (u), exponents off by t = 2^-24 (d max(scale |q|.|k|) + 8), sums in fp32 whatever their order."""
import math

import numpy as np
import pytest

from tests.test_gpu_prompt import DEV, TINY, _mods, draw

pytestmark = pytest.mark.gpu
BAD = {"nan": math.nan, "inf": math.inf, "-inf": -math.inf}


def seen_by(torch, nq, nk, window, sinks):
    j, p = torch.arange(nk, device=DEV), torch.arange(nq, device=DEV)[:, None] + nk - nq
    return (j <= p) & ((p - j < window) | (j < sinks))


def reference(torch, q, k, v, do, scale, window, sinks):
    """One sequence, 64 bits: q, do [nq][H][d], k, v [nk][Hk][d].  Values, and (after a bar) the sums that bounds need."""
    q, k, v, do = (x.double() for x in (q, k, v, do))
    (nq, H, d), (nk, Hk, _) = q.shape, k.shape
    g = H // Hk
    seen = seen_by(torch, nq, nk, window, sinks)
    kh, vh = (x.repeat_interleave(g, 1).permute(1, 0, 2).contiguous() for x in (k, v))       # [H][nk][d]
    qh, dh = (x.permute(1, 0, 2).contiguous() for x in (q, do))
    kt, vt = kh.transpose(1, 2).contiguous(), vh.transpose(1, 2).contiguous()
    w = torch.where(seen, qh @ kt * scale, -math.inf)
    size = float((qh.abs() @ kt.abs()).amax()) * scale if w.numel() else 0.0
    lse = torch.logsumexp(w, -1) if nk else torch.full((H, nq), -math.inf, dtype=torch.float64, device=DEV)
    p = torch.where(seen, torch.exp(w - torch.where(lse == -math.inf, 0.0, lse)[..., None]), 0.0)
    out = p @ vh
    rows = lambda x: x.permute(1, 0, 2)  # noqa: E731
    keys = lambda x: rows(x).reshape(nk, Hk, g, d).sum(2)  # noqa: E731
    dp, delta = dh @ vt, (dh * out).sum(-1, keepdim=True)
    far = dh.abs() @ vt.abs() + (dh * out).abs().sum(-1, keepdim=True)
    gr = p * (dp - delta)
    pt, gt = p.transpose(1, 2).contiguous(), gr.transpose(1, 2).contiguous()
    r = {"lse": lse, "out": rows(out), "out|": rows(p @ vh.abs()), "size": size, "dv": keys(pt @ dh), "dv|": keys(pt @ dh.abs()),
         "dq": rows(gr @ kh) * scale, "dk": keys(gt @ qh) * scale}
    for name, x in (("g", gr.abs()), ("p", p * far)):
        r["dq|" + name] = rows(x @ kh.abs()) * scale
        r["dk|" + name] = keys(x.transpose(1, 2).contiguous() @ qh.abs()) * scale
    return r


def check(torch, got, want, dtype, d, what="", rows=None, keys=None):
    """rows, keys: which to look at (all)."""
    u = torch.finfo(dtype).eps / 2
    t = 2.0 ** -24 * (d * want["size"] + 8)
    ud = 0.0 if dtype == torch.float32 else 2.0 ** -16
    bound = {"out": u * want["out"].abs() + (u + t) * want["out|"], "lse": 2.0 ** -24 * (d * want["size"] + 8 + want["lse"].abs()),
             "dv": u * want["dv"].abs() + (u + 2 * t) * want["dv|"]}
    for x in ("dq", "dk"):
        bound[x] = u * want[x].abs() + (u + 2 * t) * want[x + "|g"] + (t + ud) * want[x + "|p"]
    for name, x in got.items():
        x, y, b = x.double(), want[name], bound[name]
        at = keys if name in ("dk", "dv") else rows
        if at is not None:
            x, y, b = (z[:, at] if name == "lse" else z[at] for z in (x, y, b))
        same = (x == y) | ((x - y).abs() <= b + TINY)
        assert bool(same.all()), f"{what} {name}: {int((~same).sum())} of {same.numel()} off, worst {((x - y).abs() - b).max().item()}"


def run(torch, P, nq, nk, H, Hk, d, dt, window, sinks, *, seed=1, spare=3, spoil=None, std=1.0):
    """Packed sequences through forward and backward, `spare` rows behind the last: per sequence (inputs, got)."""
    Tq, Tk = sum(nq) + spare, sum(nk) + spare
    q, do = draw(torch, (Tq, H, d), dt, seed, std), draw(torch, (Tq, H, d), dt, seed + 3)
    k, v = draw(torch, (Tk, Hk, d), dt, seed + 1, std), draw(torch, (Tk, Hk, d), dt, seed + 2)
    if spoil:
        spoil(q, k, v, do)
    qs, ks = (torch.tensor(np.cumsum([0] + n), dtype=torch.int32, device=DEV) for n in (nq, nk))
    at = dict(q_start=qs, k_start=ks, window=window, sinks=sinks)
    out = torch.full((Tq, H, d), 7.0, dtype=dt, device=DEV)
    out, lse, left = P.prompt_attention(q, k, v, out=out, rest=True, **at)
    to = [torch.full(s, 7.0, dtype=dt, device=DEV) for s in ((Tq, H, d), (Tk, Hk, d), (Tk, Hk, d))]
    dq, dk, dv = P.prompt_attention_backward(do, q, k, v, out, lse, rest=left, dq=to[0], dk=to[1], dv=to[2], **at)
    torch.cuda.synchronize()
    if spare:
        assert all(bool((x[-spare:] == 0.0).all()) for x in (out, dq, dk, dv)) and bool((lse[:, -spare:] == -math.inf).all())
    a = b = 0
    for n, m in zip(nq, nk):
        i, j = slice(a, a + n), slice(b, b + m)
        yield (q[i], k[j], v[j], do[i]), dict(out=out[i], lse=lse[:, i], dq=dq[i], dk=dk[j], dv=dv[j])
        a, b = a + n, b + m


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("nq,nk,window,sinks", [(700, 690, 50, 4), (900, 200, 20, 2), (1500, 1499, 1, 40), (600, 3, 2, 2)])
def test_many_queries_of_which_the_first_see_nothing(nq, nk, window, sinks, d, dtype):
    """Their rows may hold anything, in tiles with queries that are behind the window of the first keys."""
    torch, P = _mods()
    dt = dtype_of(torch, dtype)
    for bad in (0.5, math.nan):

        def spoil(q, k, v, do):
            q[:nq - nk], do[:nq - nk] = bad, bad

        (x, got), = run(torch, P, [nq], [nk], 8, 2, d, dt, window, sinks, spoil=spoil)
        x[0][:nq - nk], x[3][:nq - nk] = 0.0, 0.0
        check(torch, got, reference(torch, *x, d ** -0.5, window, sinks), dt, d)
        assert bool((got["out"][:nq - nk] == 0).all()) and bool((got["dq"][:nq - nk] == 0).all()) and bool((got["lse"][:, :nq - nk] == -math.inf).all())


def dtype_of(torch, name):
    return torch.bfloat16 if name == "bf16" else torch.float32


WINDOWS = [(1, 0), (1, 2), (5, 0), (32, 4), (33, 33), (64, 0), (100, 1), (150, 130), (4000, 0), (2, 4000), (1 << 40, 1 << 40)]
LENGTHS = [([1, 0, 2, 0, 33], [1, 0, 2, 0, 33]), ([31, 32, 33, 63, 64, 65], [31, 32, 33, 63, 64, 65]), ([127, 128, 129, 257], [127, 128, 129, 257]),
           ([1, 5, 64, 130], [200, 5, 165, 513]),             # a prefix that is there already
           ([40, 3, 130, 7, 0], [10, 0, 129, 1, 17])]         # first queries that see nothing, sequences without keys and without queries


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("window,sinks", WINDOWS)
def test_packed_sequences(window, sinks, d, dtype):
    torch, P = _mods()
    dt = dtype_of(torch, dtype)
    for lengths in LENGTHS:
        for n, (x, got) in enumerate(run(torch, P, *lengths, 6, 2, d, dt, window, sinks)):
            check(torch, got, reference(torch, *x, d ** -0.5, window, sinks), dt, d, what=f"{lengths} sequence {n}")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("H,Hk,d", [(8, 2, 64), (16, 16, 128), (64, 32, 64), (64, 64, 128), (16, 1, 128)])
@pytest.mark.parametrize("window,sinks", [(1, 1), (70, 4), (129, 0), (300, 40), (40, 200)])
def test_first_keys_of_long_sequences(window, sinks, H, Hk, d, dtype):
    """Queries behind the window cut into chunks, waves that share rows and blocks of 128."""
    torch, P = _mods()
    dt = dtype_of(torch, dtype)
    for n, (x, got) in enumerate(run(torch, P, [700, 1, 0, 40, 515, 290], [700, 1, 30, 90, 900, 290], H, Hk, d, dt, window, sinks)):
        check(torch, got, reference(torch, *x, d ** -0.5, window, sinks), dt, d, what=f"sequence {n}")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("window,sinks", [(3, 1), (20, 0), (60, 7)])
def test_more_sequences_than_a_wave_has_lanes(window, sinks, dtype):
    torch, P = _mods()
    dt = dtype_of(torch, dtype)
    lengths = [int(x) for x in np.random.default_rng(5).integers(0, 40, 150)]
    lengths[70], lengths[140] = 290, 333
    for n, (x, got) in enumerate(run(torch, P, lengths, lengths, 4, 1, 64, dt, window, sinks)):
        check(torch, got, reference(torch, *x, 64 ** -0.5, window, sinks), dt, 64, what=f"sequence {n}")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("B,H,Hk,nq,nk,d,window,sinks", [(2, 4, 2, 100, 100, 64, 17, 2), (1, 2, 2, 1, 1000, 128, 100, 4), (3, 2, 1, 129, 200, 128, 64, 0),
                                                         (2, 3, 3, 64, 40, 64, 10, 1), (2, 8, 2, 777, 777, 64, 130, 5), (3, 8, 4, 600, 700, 128, 1, 33)])
def test_dense_batches(B, H, Hk, nq, nk, d, window, sinks, dtype):
    torch, P = _mods()
    dt = dtype_of(torch, dtype)
    q, do = draw(torch, (B, H, nq, d), dt, 1), draw(torch, (B, nq, H, d), dt, 4).transpose(1, 2)     # another order of dimensions
    kv = draw(torch, (B, 2 * Hk, nk, d), dt, 2)
    k, v = kv[:, :Hk], kv[:, Hk:]
    how = dict(window=window, sinks=sinks)
    out, lse, rest = P.prompt_attention(q, k, v, rest=True, **how)
    dq, dk, dv = P.prompt_attention_backward(do, q, k, v, out, lse, rest=rest, **how)
    for b in range(B):
        want = reference(torch, *(x[b].transpose(0, 1) for x in (q, k, v, do)), d ** -0.5, window, sinks)
        got = dict(out=out[b].transpose(0, 1), lse=lse[b], dq=dq[b].transpose(0, 1), dk=dk[b].transpose(0, 1), dv=dv[b].transpose(0, 1))
        check(torch, got, want, dt, d, what=f"sequence {b}")


def test_a_window_that_hides_nothing_is_plain_attention():
    """Outputs equal to the bit (the same tiles in the same order), gradients of both within their bounds of the definition's (sums in
    another order: two results within a bound of a third are within two of each other, and no nearer need be)."""
    torch, P = _mods()
    for dt in (torch.bfloat16, torch.float32):
        q, k, v, do = (draw(torch, (2, h, 300, 64), dt, s) for h, s in ((4, 1), (2, 2), (2, 3), (4, 4)))
        want = P.prompt_attention(q, k, v, rest=True)
        exact = [reference(torch, *(x[b].transpose(0, 1) for x in (q, k, v, do)), 64 ** -0.5, 300, 0) for b in range(2)]
        for how in ({}, dict(window=300), dict(window=1 << 31), dict(window=1, sinks=300), dict(window=300, sinks=300)):
            got = P.prompt_attention(q, k, v, rest=True, **how)
            assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
            grads = P.prompt_attention_backward(do, q, k, v, got[0], got[1], rest=got[2], **how)
            for b in range(2):
                check(torch, {n: x[b].transpose(0, 1) for n, x in zip(("dq", "dk", "dv"), grads)}, exact[b], dt, 64, what=str(how))


@pytest.mark.parametrize("std,scale", [(8.0, None), (1.0, 1.0), (1e-4, None)])
def test_sharp_and_flat_weights(std, scale):
    torch, P = _mods()
    for dt in (torch.bfloat16, torch.float32):
        q, k, v, do = (draw(torch, (333, h, 128), dt, s, z) for h, s, z in ((2, 1, std), (1, 2, std), (1, 3, 1.0), (2, 4, 1.0)))
        at = dict(q_start=torch.tensor([0, 333], dtype=torch.int32, device=DEV), k_start=torch.tensor([0, 333], dtype=torch.int32, device=DEV),
                  scale=scale, window=77, sinks=3)
        out, lse, rest = P.prompt_attention(q, k, v, rest=True, **at)
        dq, dk, dv = P.prompt_attention_backward(do, q, k, v, out, lse, rest=rest, **at)
        check(torch, dict(out=out, lse=lse, dq=dq, dk=dk, dv=dv), reference(torch, q, k, v, do, scale or 128 ** -0.5, 77, 3), dt, 128)


HIDDEN = [  # queries, keys, window, sinks, heads, kv heads
    (200, 200, 30, 3, 4, 2), (300, 300, 64, 0, 4, 2), (257, 257, 100, 70, 4, 2), (260, 400, 40, 5, 4, 2), (700, 700, 90, 4, 8, 2), (384, 384, 33, 1, 64, 64)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("bad", list(BAD))
@pytest.mark.parametrize("nq,nk,window,sinks,H,Hk", HIDDEN)
def test_keys_that_a_query_does_not_see_may_hold_anything(nq, nk, window, sinks, H, Hk, bad, dtype):
    torch, P = _mods()
    d, dt = 64, dtype_of(torch, dtype)
    for row in (0, sinks, window - 1, nk // 3, nk // 2 + 7):

        def spoil(q, k, v, do):
            k[row], v[row] = BAD[bad], BAD[bad]

        (x, got), = run(torch, P, [nq], [nk], H, Hk, d, dt, window, sinks, spoil=spoil)
        x[1][row], x[2][row] = 0.0, 0.0
        want = reference(torch, *x, d ** -0.5, window, sinks)
        blind = ~seen_by(torch, nq, nk, window, sinks)[:, row]
        check(torch, {n: got[n] for n in ("out", "lse", "dq")}, want, dt, d, what=f"key {row}", rows=blind)
        if bad == "nan":
            assert bool(torch.isnan(got["out"][~blind]).all()) and bool(torch.isnan(got["dq"][~blind]).all())
        if bool(blind.all()):        # nobody sees it: it is not there
            assert bool((got["dk"][row] == 0).all()) and bool((got["dv"][row] == 0).all())
            others = torch.arange(nk, device=DEV) != row
            check(torch, {n: got[n] for n in ("dk", "dv")}, want, dt, d, what=f"key {row}", keys=others)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("bad", list(BAD))
@pytest.mark.parametrize("nq,nk,window,sinks,H,Hk", HIDDEN)
def test_queries_reach_no_key_that_they_do_not_see(nq, nk, window, sinks, H, Hk, bad, dtype):
    torch, P = _mods()
    d, dt = 64, dtype_of(torch, dtype)
    for row in (0, 1, window, nq // 2, nq - 1):

        def spoil(q, k, v, do):
            q[row], do[row] = BAD[bad], BAD[bad]

        (x, got), = run(torch, P, [nq], [nk], H, Hk, d, dt, window, sinks, spoil=spoil)
        x[0][row], x[3][row] = 0.0, 0.0
        want = reference(torch, *x, d ** -0.5, window, sinks)
        unseen = ~seen_by(torch, nq, nk, window, sinks)[row]
        check(torch, {n: got[n] for n in ("dk", "dv")}, want, dt, d, what=f"query {row}", keys=unseen)
        check(torch, {n: got[n] for n in ("out", "lse", "dq")}, want, dt, d, what=f"query {row}", rows=torch.arange(nq, device=DEV) != row)
        if bad == "nan":
            assert bool(torch.isnan(got["dk"][~unseen]).all()) and bool(torch.isnan(got["dv"][~unseen]).all())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_gradients_against_differences(dtype):
    """sum(d_out . out) along a direction, by central differences of the forward pass in fp32: h = 2^-6 leaves h^2 / 6 of the third
    derivative (4e-5 of its size, at most some tens here) and 2 sqrt(n) 2^-24 / h of rounding."""
    torch, P = _mods()
    d, n = 64, 90
    at = dict(q_start=torch.tensor([0, 20, n], dtype=torch.int32, device=DEV), k_start=torch.tensor([0, 20, n], dtype=torch.int32, device=DEV),
              window=13, sinks=2)
    dt = dtype_of(torch, dtype)
    q, k, v, do = (draw(torch, (n, h, d), dt, s, 0.5) for h, s in ((4, 1), (2, 2), (2, 3), (4, 4)))
    out, lse, rest = P.prompt_attention(q, k, v, rest=True, **at)
    grads = P.prompt_attention_backward(do, q, k, v, out, lse, rest=rest, **at)
    wide = [x.float() for x in (q, k, v)]

    def loss(a, b, c):
        return float((P.prompt_attention(a, b, c, **at)[0].double() * do.double()).sum())

    h = 2.0 ** -6
    for i, x in enumerate(wide):
        u = draw(torch, x.shape, torch.float32, 50 + i)
        hi, lo = list(wide), list(wide)
        hi[i], lo[i] = x + h * u, x - h * u
        slope = (loss(*hi) - loss(*lo)) / (2 * h)
        want = float((grads[i].double() * u.double()).sum())
        size = float((grads[i].double() * u.double()).square().sum().sqrt())       # of a sum of independent terms
        assert abs(slope - want) < 0.02 * size + 1e-3, (i, slope, want, size)


def test_autograd_takes_the_window_along():
    torch, P = _mods()
    q, k, v, do = (draw(torch, (150, h, 64), torch.bfloat16, s) for h, s in ((4, 1), (2, 2), (2, 3), (4, 4)))
    at = dict(q_start=torch.tensor([0, 150], dtype=torch.int32, device=DEV), k_start=torch.tensor([0, 150], dtype=torch.int32, device=DEV), window=20, sinks=1)
    out, lse, rest = P.prompt_attention(q, k, v, rest=True, **at)
    want = P.prompt_attention_backward(do, q, k, v, out, lse, rest=rest, **at)
    leaves = [x.clone().requires_grad_() for x in (q, k, v)]
    got, _, _ = P.prompt_attention(*leaves, rest=True, **at)
    assert torch.equal(got, out)
    got.backward(do)
    for x, y in zip(leaves, want):
        assert torch.equal(x.grad, y)


def test_equal_inputs_give_equal_bits_and_a_graph_replays():
    torch, P = _mods()
    dt, d, n = torch.bfloat16, 128, [300, 17, 529]
    T = sum(n)
    q, k, v, do = (draw(torch, (T, h, d), dt, s) for h, s in ((8, 1), (2, 2), (2, 3), (8, 4)))
    starts = torch.tensor(np.cumsum([0] + n), dtype=torch.int32, device=DEV)
    at = dict(q_start=starts, k_start=starts, window=65, sinks=4)

    def all_of_it():
        out, lse, rest = P.prompt_attention(q, k, v, rest=True, **at)
        return (out, lse, rest, *P.prompt_attention_backward(do, q, k, v, out, lse, rest=rest, **at))

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


def test_rows_in_front_of_the_first_sequence():
    torch, P = _mods()
    dt, d, front = torch.bfloat16, 64, 37
    q, k, v, do = (draw(torch, (900, h, d), dt, s) for h, s in ((8, 1), (2, 2), (2, 3), (8, 4)))
    starts = torch.tensor([front, front + 600, front + 840], dtype=torch.int32, device=DEV)
    at = dict(q_start=starts, k_start=starts, window=50, sinks=2)
    out, lse, rest = P.prompt_attention(q, k, v, rest=True, **at)
    dq, dk, dv = P.prompt_attention_backward(do, q, k, v, out, lse, rest=rest, **at)
    for x in (out, dq, dk, dv):
        assert bool((x[:front] == 0).all()) and bool((x[front + 840:] == 0).all())
    for i in (slice(front, front + 600), slice(front + 600, front + 840)):
        want = reference(torch, q[i], k[i], v[i], do[i], d ** -0.5, 50, 2)
        check(torch, dict(out=out[i], lse=lse[:, i], dq=dq[i], dk=dk[i], dv=dv[i]), want, dt, d)
