"""Forward-mode derivatives, which neither attention nor rotation has: a tensor with a tangent is refused, and not answered without one.  Tensors here lie
on the host and say that they are on a device."""
import pytest
import torch
from torch.autograd import forward_ad

from paper_2407_02328_amd import Rotary, WindowCache, binding, prompt_attention, prompt_attention_backward, rotate_heads, rotate_heads_backward
from tests.test_devices_cpu import Machine, OnGpu, on_gpu


@pytest.fixture
def machine(monkeypatch):
    m = Machine()
    m.adore_rotary_turns = lambda *a: 0
    empty, strided = torch.empty, torch.empty_strided
    monkeypatch.setattr(binding, "load_library", lambda: m)
    monkeypatch.setattr(binding, "_stream", lambda index: 0)
    monkeypatch.setattr(binding, "_current", lambda: m.current, raising=False)
    monkeypatch.setattr(torch.cuda, "device", m.device)
    monkeypatch.setattr(torch, "empty", lambda *args, device=None, **kw: empty(*args, **kw).as_subclass(OnGpu))
    monkeypatch.setattr(torch, "empty_strided", lambda *args, device=None, **kw: strided(*args, **kw).as_subclass(OnGpu))
    monkeypatch.setattr(Rotary, "on", lambda self, device: 64)
    return m


def dual(t):
    return forward_ad.make_dual(t.as_subclass(torch.Tensor), torch.ones_like(t.as_subclass(torch.Tensor))).as_subclass(OnGpu)


def ring():
    cache = on_gpu((2 * 2 * 2 * 64 * 64 + 128,))
    at = -cache.data_ptr() % 256 // 2
    return WindowCache(batch=2, heads=4, kv_heads=2, head_dim=64, window=60, sinks=4, dtype="bf16", cursor=on_gpu((2, 2), torch.int32),
                       cache=cache[at:at + 2 * 2 * 2 * 64 * 64].view(2, 2, 2, 64 * 64))


def refusals():
    """Calls, and their tensors that may have a tangent, in a list that the test puts them into."""
    q, k, pos, w = on_gpu((5, 4, 64)), on_gpu((5, 2, 64)), on_gpu((5,), torch.int32), on_gpu((64,), torch.float32)
    rotary = Rotary(64)
    yield [q, k, w], lambda q, k, w: rotate_heads(q, k, pos, rotary, q_weight=w, k_weight=w)
    yield [q, k, w], lambda q, k, w: rotate_heads(q, k, pos, rotary, q_weight=w, k_weight=w, q_out=on_gpu((5, 4, 64)), k_out=on_gpu((5, 2, 64)))
    yield [q], lambda q: rotate_heads(q, None, pos, rotary)
    yield [q, k, q, k, w], lambda dq, dk, q, k, w: rotate_heads_backward(dq, dk, q, k, pos, rotary, q_weight=w, k_weight=w)
    b, c = on_gpu((2, 4, 5, 64)), on_gpu((2, 2, 5, 64))
    lse = on_gpu((2, 4, 5), torch.float32)
    for how in ({}, dict(window=3, sinks=1)):
        yield [b, c, c], lambda q, k, v, how=how: prompt_attention(q, k, v, **how)
        yield [b, c, c], lambda q, k, v, how=how: prompt_attention(q, k, v, out=on_gpu((2, 4, 5, 64)), **how)
        yield [b, b, c, c, b], lambda d, q, k, v, out, how=how: prompt_attention_backward(d, q, k, v, out, lse, **how)
    cache = ring()
    yield [c, c], lambda k, v: cache.fill(k, v)
    yield [on_gpu((2, 4, 64)), on_gpu((2, 2, 64)), on_gpu((2, 2, 64))], lambda q, k, v: cache.step(q, k, v)


def test_tangents_are_refused(machine):
    for tensors, call in refusals():
        call(*tensors)
        n = len(machine.calls)
        with forward_ad.dual_level():
            call(*tensors)                               # (none of them has one)
            assert len(machine.calls) == n + 1
            for i in range(len(tensors)):
                with pytest.raises((ValueError, NotImplementedError)):
                    call(*(dual(t) if i == j else t for j, t in enumerate(tensors)))
        assert len(machine.calls) == n + 1
        machine.calls.clear()


def test_a_tangent_is_refused_where_gradients_are_required_too(machine):
    q, pos = on_gpu((5, 4, 64), torch.float32), on_gpu((5,), torch.int32)
    w = torch.ones(64).as_subclass(OnGpu).requires_grad_()
    with forward_ad.dual_level():
        with pytest.raises((ValueError, NotImplementedError)):
            rotate_heads(dual(q), None, pos, Rotary(64), q_weight=w)
    assert not [c for c in machine.calls if c[0] == "adore_rotate_heads"]
