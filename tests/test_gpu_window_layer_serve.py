"""examples/window_layer.py: serving needs the prompts' keys and values, and not their attention."""
import pytest

from tests.test_gpu_ring import _mods
from tests.test_gpu_window_layer import made

pytestmark = pytest.mark.gpu


def test_prompts_are_loaded_without_their_attention():
    torch, _ = _mods()
    from examples.window_layer import DEV, packed, serve
    layer = made(torch)
    start, positions = packed([70, 1, 33])
    g = torch.Generator(device=DEV)
    g.manual_seed(3)
    x = torch.randn((104, 256), generator=g, device=DEV).bfloat16()
    following = torch.randn((5, 3, 256), generator=g, device=DEV).bfloat16()
    cache, outs = serve(layer, x, start, positions, following)
    layer.attend = None
    again, same = serve(layer, x, start, positions, following)
    assert torch.equal(outs, same) and all(torch.equal(a, b) for a, b in zip(cache.read(), again.read()))
