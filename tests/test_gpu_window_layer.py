"""Rotation, attention with a window and the ring together, as a layer is trained and served with them (examples/window_layer.py)."""
import math

import pytest

from tests.test_gpu_ring import _mods, draw
from tests.test_gpu_window import reference

pytestmark = pytest.mark.gpu


def made(torch, **kw):
    from examples.window_layer import Layer
    return Layer(**dict(dict(hidden=256, heads=8, kv_heads=2, head_dim=64, window=20, sinks=3), **kw))


@pytest.mark.parametrize("window,sinks", [(20, 3), (1, 0), (500, 0), (16, 40)])
def test_a_token_at_a_time_is_the_prompt_at_once(window, sinks):
    """The rows that the ring holds are those of the prompts' pass to the bit (each is projected with its batch, normed and rotated by
    itself; projections of other batches are rounded apart, so that these are handed in), and outputs are within the bounds of
    test_gpu_window.py and test_gpu_ring.py of the definition."""
    torch, P = _mods()
    from examples.window_layer import packed
    H, Hk, d, lengths, T = 8, 2, 64, [70, 1, 33], 30
    rotary = P.Rotary(d, base=500000.0, factor=4.0, original=32.0)
    w = 1.0 + 0.2 * draw(torch, (d,), torch.float32, 9)
    for dtype, dt in (("bf16", torch.bfloat16), ("f32", torch.float32)):
        u = torch.finfo(dt).eps / 2
        rows = [draw(torch, (n + T, H + 2 * Hk, d), dt, 3 + n) for n in lengths]
        start, positions = packed(lengths)
        prompt = torch.cat([x[:n] for x, n in zip(rows, lengths)])
        q, k = P.rotate_heads(prompt[:, :H], prompt[:, H:H + Hk], positions, rotary, q_weight=w, k_weight=w)
        P.prompt_attention(q, k, prompt[:, H + Hk:], q_start=start, k_start=start, window=window, sinks=sinks)
        cache = P.WindowCache(batch=3, heads=H, kv_heads=Hk, head_dim=d, window=window, sinks=sinks, dtype=dt)
        cache.fill(k, prompt[:, H + Hk:], k_start=start)
        outs = []
        for t in range(T):
            x = torch.stack([r[n + t] for r, n in zip(rows, lengths)])
            qt, kt = P.rotate_heads(x[:, :H], x[:, H:H + Hk], cache.positions, rotary, q_weight=w, k_weight=w)
            outs.append(cache.step(qt, kt, x[:, H + Hk:].contiguous()))
        held_k, held_v = cache.read()
        for b, (r, n) in enumerate(zip(rows, lengths)):
            at, pos = packed([n + T])
            q, k = P.rotate_heads(r[:, :H], r[:, H:H + Hk], pos, rotary, q_weight=w, k_weight=w)
            v = r[:, H + Hk:]
            kept = list(range(n + T)) if n + T <= window + sinks else list(range(sinks)) + list(range(n + T - window, n + T))
            assert torch.equal(held_k[b, :, :len(kept)], k[kept].transpose(0, 1)) and torch.equal(held_v[b, :, :len(kept)], v[kept].transpose(0, 1))
            want = reference(torch, q, k, v, q, d ** -0.5, window, sinks)
            t = 2.0 ** -24 * (d * want["size"] + 8 + window + sinks)
            term = 2.0 ** -16 if dt == torch.bfloat16 else 2.0 ** -22
            got = torch.stack(outs)[:, b].double()
            bound = u * want["out"][n:].abs() + (t + term) * want["out|"][n:]
            assert bool(((got - want["out"][n:]).abs() <= bound).all()), (dtype, b)
            whole = P.prompt_attention(q, k, v, q_start=at, k_start=at, window=window, sinks=sinks)[0][n:].double()
            assert bool(((got - whole).abs() <= 2 * bound + (u + t) * want["out|"][n:]).all()), (dtype, b)


def test_gradients_of_the_layer():
    """A step's gradients by torch's autograd through the projection, the rotation and the attention, against those of the same layer in
    64 bits (elementary operations, weights and inputs as they are).  Every tensor on the way is rounded to bf16 once, forward and
    backward: less than 16 roundings of 2^-9 each of its norm, some of which the softmax doubles."""
    torch, P = _mods()
    from examples.window_layer import packed
    layer = made(torch)
    start, positions = packed([70, 1, 133])
    x = draw(torch, (204, 256), torch.bfloat16, 3)
    d_y = draw(torch, (204, 256), torch.bfloat16, 4)
    for w in layer.parameters():
        w.requires_grad_(True)
    layer(x, start, positions).backward(d_y)
    W = [w.detach().double().requires_grad_(True) for w in layer.parameters()]
    H, Hk, d = layer.heads, layer.kv_heads, layer.head_dim
    qkv = (x.double() @ W[0]).unflatten(-1, (-1, d))
    t = positions.double()[:, None] * 10000.0 ** (-2.0 * torch.arange(d // 2, device=x.device, dtype=torch.float64) / d)
    c, s = t.cos()[:, None], t.sin()[:, None]

    def turned(y, w):
        y = y / (y.square().mean(-1, keepdim=True) + 1e-6).sqrt() * w
        a, b = y.split(d // 2, -1)
        return torch.cat([a * c - b * s, a * s + b * c], -1)

    q, k, v = turned(qkv[:, :H], W[2]), turned(qkv[:, H:H + Hk], W[3]), qkv[:, H + Hk:]
    outs = []
    for i, j in ((0, 70), (70, 71), (71, 204)):
        kk, vv = (y[i:j].repeat_interleave(H // Hk, 1).permute(1, 0, 2).contiguous() for y in (k, v))
        n = torch.arange(j - i, device=x.device)
        far = n[:, None] - n
        seen = (far >= 0) & ((far < layer.window) | (n < layer.sinks))
        p = torch.softmax(torch.where(seen, q[i:j].permute(1, 0, 2).contiguous() @ kk.transpose(1, 2).contiguous() * d ** -0.5, -math.inf), -1)
        outs.append((p @ vv).permute(1, 0, 2))
    (torch.cat(outs).flatten(1) @ W[1]).backward(d_y.double())
    for got, want in zip(layer.parameters(), W):
        off = float((got.grad.double() - want.grad).norm() / want.grad.norm())
        assert off < 32 * 2.0 ** -9, off


def test_the_example_runs():
    torch, _ = _mods()
    from examples.window_layer import DEV, all_at_once, packed, serve, train
    layer, lengths = made(torch), [70, 1, 33]
    g = torch.Generator(device=DEV)
    g.manual_seed(3)
    x = torch.randn((sum(lengths), 256), generator=g, device=DEV).bfloat16()
    start, positions = packed(lengths)
    losses = train(layer, x, x.float().roll(1, 0), start, positions, 3, 2.0)
    assert all(math.isfinite(v) for v in losses)
    following = torch.randn((40, 3, 256), generator=g, device=DEV).bfloat16()
    cache, outs = serve(layer, x, start, positions, following)
    want = all_at_once(layer, x, start, following).float()
    # products of other batches are rounded apart, 2^-9 of an element of q, k and v each, and the weights once: a few of those roundings
    assert float((outs.float() - want).norm() / want.norm()) < 8 * 2.0 ** -8
    assert cache.positions.tolist() == [n + 40 for n in lengths]
