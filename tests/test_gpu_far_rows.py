"""Rows whose offsets pass 32 bits: packed prompts at the end of tensors of 5 GB, and the last rows of a cache in 4 bits of 4.5 GB."""
import pytest

from tests.test_gpu_prompt import DEV, _mods, check, draw, reference

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("H,Hk", [(32, 32), (32, 2)])
def test_prompts_at_the_end_of_large_tensors(H, Hk):
    torch, P = _mods()
    T, n, m, d, dt = 600_000, 200, 150, 128, torch.bfloat16
    Tk = T if Hk == H else 9_000_000
    assert T * H * d > 2 ** 31 and Tk * Hk * d > 2 ** 31
    q, k, v, do = (torch.empty((t, h, d), dtype=dt, device=DEV) for t, h in ((T, H), (Tk, Hk), (Tk, Hk), (T, H)))
    for i, x in enumerate((q, k, v, do)):
        x[-n - m:] = draw(torch, (n + m,) + x.shape[1:], dt, 1 + i)
    at = dict(q_start=torch.tensor([T - n - m, T - m, T], dtype=torch.int32, device=DEV),
              k_start=torch.tensor([Tk - n - m, Tk - m, Tk], dtype=torch.int32, device=DEV))
    out, lse, rest = P.prompt_attention(q, k, v, rest=True, **at)
    dq, dk, dv = P.prompt_attention_backward(do, q, k, v, out, lse, rest=rest, **at)
    scores = P.prompt_scores(q, k, lse, **at)
    for i in (slice(-n - m, -m), slice(-m, None)):
        want = reference(torch, q[i], k[i], v[i], do[i], d ** -0.5)
        check(torch, dict(out=out[i], lse=lse[:, i], scores=scores[:, i], dq=dq[i], dk=dk[i], dv=dv[i]), want, dt, d)


def test_the_last_rows_of_a_large_cache():
    torch, P = _mods()
    B, H, K, d, dt = 64, 32, 16384, 128, torch.bfloat16
    shape = dict(heads=H, kv_heads=H, head_dim=d, slots=K, recent=16, dtype=dt)
    big, one = P.Q4Cache(batch=B, **shape), P.Q4Cache(batch=1, **shape)
    assert big.cache.numel() > 2 ** 32
    k, v = draw(torch, (1, H, K + 100, d), dt, 1), draw(torch, (1, H, K + 100, d), dt, 2)
    one.fill(k, v, draw(torch, (1, H, K + 100), torch.float32, 3).abs())
    names = ("cache", "slot_pos", "score", "cursor")
    for name in names:
        getattr(big, name)[-1:] = getattr(one, name)
    assert all(torch.equal(x[-1:], y) for x, y in zip(big.read(), one.read()))
    for i in range(2):
        q, k, v = (draw(torch, (B, H, d), dt, 10 * i + j) for j in range(3))
        out, k_held, v_held = big.step(q, k, v, held=True)
        want, k_one, v_one = one.step(*(x[-1:].contiguous() for x in (q, k, v)), held=True)
        assert torch.equal(k_held[-1:], k_one) and torch.equal(v_held[-1:], v_one)
        assert torch.equal(big.cache[-1:], one.cache) and torch.equal(big.slot_pos[-1:], one.slot_pos)
        # Two cuts of one sum: outputs are rounded once each (2^-8 together), weights of some 10 units of exponent are off by 2^-24 times
        # 128 products and 16384 terms at most, on each side
        off = 2.0 ** -8 * want.float().abs() + 2.0 ** -9
        assert bool(((out[-1:].float() - want.float()).abs() <= off).all())
        assert bool(((big.score[-1:] - one.score).abs() <= 2.0 ** -9 * (one.score.abs() + 2.0 ** -14)).all())
        for name in ("score", "cursor"):                 # (where the smallest scores are within that, the next slots may differ)
            getattr(big, name)[-1:] = getattr(one, name)
