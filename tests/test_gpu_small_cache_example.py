"""The example that trains a layer with prompt attention and serves it from the cache in 4 bits, on a few short prompts."""
import pytest

pytestmark = pytest.mark.gpu


def test_training_and_serving_run_together():
    import torch
    from examples.small_cache import DEV, Layer, full_attention, serve, starts_of, train
    g = torch.Generator(device=DEV)
    g.manual_seed(3)
    layer, lengths = Layer(hidden=256, heads=8, kv_heads=2, head_dim=64), [70, 1, 33]
    x = torch.randn((sum(lengths), 256), generator=g, device=DEV).bfloat16()
    start = starts_of(lengths)
    losses = train(layer, x, x.float().roll(1, 0), start, 10, 2.0)
    assert losses[-1] < losses[0]
    following = torch.randn((20, 3, 256), generator=g, device=DEV).bfloat16()
    # Room for everything: what rounding to 4 bits leaves.  A row of normal elements is off by 0.112 of its norm, and so is an average of rows
    # of V; exponents are off by 0.112 (unit normal q), which moves the average as far again: 0.16 together.
    cache, outs = serve(layer, x, start, following, 96, 8)
    want = full_attention(layer, x, start, following).float()
    assert float((outs.float() - want).norm() / want.norm()) < 0.25
    assert bool((cache.cursor[..., 1] == torch.tensor(lengths, device=DEV)[:, None] + 20).all())
    # half the room: every slot is taken, the last tokens are all there
    cache, outs = serve(layer, x, start, following, 40, 8)
    assert bool(torch.isfinite(outs).all())
    for b, n in enumerate(lengths):
        pos = cache.slot_pos[b].sort(-1)[0]
        assert bool((pos[:, -8:] == torch.arange(n + 12, n + 20, device=DEV)).all())
        assert bool((pos >= 0).sum() == 2 * min(40, n + 20))
