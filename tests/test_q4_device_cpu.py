"""A cache on a device that is named without its number."""
import torch

from paper_2407_02328_amd import Q4Cache
from tests.test_devices_cpu import OnGpu, machine, on_gpu  # noqa: F401


def test_a_device_without_a_number(machine, monkeypatch):  # noqa: F811
    monkeypatch.setattr(OnGpu, "index", 0)
    shape = dict(batch=2, heads=4, kv_heads=2, head_dim=64, slots=64, recent=8, dtype="bf16", device="cuda")
    cache = Q4Cache(**shape)
    assert cache.device == torch.device("cuda", 0)
    k = on_gpu((2, 2, 5, 64))
    cache.fill(k, k)
    cache.step(on_gpu((2, 4, 64)), on_gpu((2, 2, 64)), on_gpu((2, 2, 64)))
    cache.read(on_gpu((2, 2, 64, 64)), on_gpu((2, 2, 64, 64)))
    assert [name for name, _ in machine.calls] == ["adore_q4_fill", "adore_q4_step", "adore_q4_read"]
    cursor = on_gpu((2, 2, 2), torch.int32)
    assert Q4Cache(**shape, cursor=cursor).cursor is cursor
