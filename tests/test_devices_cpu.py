"""Which device the calls on prompts and on a cache in 4 bits take place on: that of their tensors, whichever is current.  Tensors here
lie on the host and say that they are on a device; the library and torch's notion of the current device are stood in for."""
import pytest
import torch

from paper_2407_02328_amd import Q4Cache, binding, prompt_attention, prompt_attention_backward, prompt_scores


class OnGpu(torch.Tensor):
    index = 1

    @property
    def device(self):
        return torch.device("cuda", self.index)

    @property
    def is_cuda(self):
        return True

    def get_device(self):
        return self.index


class Machine:
    """The current device, and the library's calls with the device each was made on."""

    def __init__(self):
        self.current, self.calls, self.switches = 0, [], 0

    def __getattr__(self, name):
        def call(*args):
            if name.endswith("_bytes"):
                return 256
            self.calls.append((name, self.current))
            return 0
        return call

    def device(self, index):
        machine = self

        class Guard:
            def __enter__(self):
                self.before, machine.current = machine.current, getattr(index, "index", index)
                machine.switches += 1

            def __exit__(self, *error):
                machine.current = self.before
        return Guard()


@pytest.fixture
def machine(monkeypatch):
    m = Machine()
    empty, full = torch.empty, torch.full
    monkeypatch.setattr(binding, "load_library", lambda: m)
    monkeypatch.setattr(binding, "_stream", lambda index: 0)
    monkeypatch.setattr(binding, "_current", lambda: m.current, raising=False)
    monkeypatch.setattr(torch.cuda, "device", m.device)
    monkeypatch.setattr(torch, "empty", lambda *args, device=None, **kw: empty(*args, **kw).as_subclass(OnGpu))
    monkeypatch.setattr(torch, "full", lambda *args, device=None, **kw: full(*args, **kw).as_subclass(OnGpu))
    return m


def on_gpu(shape, dtype=torch.bfloat16):
    return torch.zeros(shape, dtype=dtype).as_subclass(OnGpu)


def every_call():
    q, k = on_gpu((2, 4, 5, 64)), on_gpu((2, 2, 5, 64))
    out, lse = prompt_attention(q, k, k)
    prompt_attention_backward(q, q, k, k, out, lse)
    prompt_scores(q, k, lse)
    cache = Q4Cache(batch=2, heads=4, kv_heads=2, head_dim=64, slots=64, recent=8, dtype="bf16", device="cuda:1")
    cache.fill(k, k)
    cache.step(on_gpu((2, 4, 64)), on_gpu((2, 2, 64)), on_gpu((2, 2, 64)))
    cache.step(on_gpu((2, 4, 64)), on_gpu((2, 2, 64)), on_gpu((2, 2, 64)), held=True)
    cache.read()
    return ["adore_prompt_attention", "adore_prompt_attention_backward", "adore_prompt_scores", "adore_q4_fill", "adore_q4_step", "adore_q4_step",
            "adore_q4_read"]


def test_calls_take_place_on_the_device_of_their_tensors(machine):
    names = every_call()
    assert machine.calls == [(name, 1) for name in names]
    assert machine.current == 0 and machine.switches == len(names)


def test_the_current_device_is_not_set_where_it_is_theirs(machine):
    machine.current = 1
    names = every_call()
    assert machine.calls == [(name, 1) for name in names] and machine.switches == 0
