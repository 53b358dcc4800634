"""Host-side checks of the window cache: sizes, and arguments that are refused before anything is enqueued."""
import ctypes

import pytest

from paper_2407_02328_amd.binding import AdoreRingConfig, AdoreRows
from tests.test_prompt_cpu import FAKE, INVALID, UNSUPPORTED, WORKSPACE, lib  # noqa: F401

GOOD = dict(batch=2, heads=4, kv_heads=2, head_dim=64, window=100, sinks=5, dtype=1, scale=0.0)


def config(**kw):
    return ctypes.byref(AdoreRingConfig(**dict(GOOD, **kw)))


def test_sizes(lib):  # noqa: F811
    assert lib.adore_ring_cache_bytes(config()) == 2 * 2 * 4 * 64 * 64 * 2
    assert lib.adore_ring_cache_bytes(config(window=27)) == 2 * 2 * 1 * 64 * 64 * 2
    assert lib.adore_ring_cache_bytes(config(window=28, dtype=0, head_dim=128)) == 2 * 2 * 2 * 64 * 128 * 4
    for kw in ({}, dict(window=20000), dict(heads=48, kv_heads=1), dict(batch=512)):
        assert lib.adore_ring_workspace_bytes(config(**kw)) >= 256
    assert lib.adore_ring_workspace_bytes(config(window=20000)) > lib.adore_ring_workspace_bytes(config())
    assert lib.adore_ring_cache_bytes(None) == 0 and lib.adore_ring_workspace_bytes(None) == 0


REFUSED = [(dict(batch=0), INVALID), (dict(heads=3), INVALID), (dict(kv_heads=0), INVALID), (dict(window=0), INVALID), (dict(window=-4), INVALID),
           (dict(sinks=-1), INVALID), (dict(dtype=3), INVALID), (dict(scale=-0.5), INVALID), (dict(scale=float("inf")), INVALID), (dict(head_dim=0), INVALID),
           (dict(head_dim=80), UNSUPPORTED), (dict(window=1 << 20), UNSUPPORTED), (dict(window=(1 << 31) - 1, sinks=(1 << 31) - 1), UNSUPPORTED),
           (dict(sinks=1 << 20), UNSUPPORTED), (dict(batch=1 << 17), UNSUPPORTED), (dict(heads=8192), UNSUPPORTED), (dict(batch=1024, window=1 << 19), UNSUPPORTED)]


def rows(**kw):
    return ctypes.byref(AdoreRows(**dict(dict(data=FAKE, seq=0, token=128, head=64), **kw)))


def calls(lib, cfg, **other):  # noqa: F811
    p = lambda name: other.get(name, FAKE)  # noqa: E731
    return (lib.adore_ring_fill(cfg, p("k_start"), other.get("tokens", 10), other.get("k_rows", rows()), other.get("v_rows", rows()), p("seen"), p("cache"),
                                p("cursor"), None),
            lib.adore_ring_step(cfg, p("q"), p("k"), p("v"), p("cache"), p("cursor"), p("out"), p("workspace"), other.get("bytes", 1 << 30), None),
            lib.adore_ring_read(cfg, p("cache"), p("cursor"), p("k"), p("v"), None))


@pytest.mark.parametrize("change,code", REFUSED)
def test_configurations_are_refused(lib, change, code):  # noqa: F811
    assert calls(lib, config(**change)) == (code,) * 3
    assert lib.adore_ring_cache_bytes(config(**change)) == 0 and lib.adore_ring_workspace_bytes(config(**change)) == 0


def test_missing_and_misplaced_buffers_are_refused(lib):  # noqa: F811
    assert calls(lib, None) == (INVALID,) * 3
    for name, off in (("cache", 128), ("cursor", 2)):
        for value in (None, FAKE + off):
            assert calls(lib, config(), **{name: value}) == (INVALID,) * 3
    bad = dict(cache=None)                           # (keeps the calls that a change does not concern from enqueuing)
    step = lambda **kw: lib.adore_ring_step(config(), *[kw.get(n, FAKE) for n in ("q", "k", "v", "cache", "cursor", "out", "workspace")],  # noqa: E731
                                            kw.get("bytes", 1 << 30), None)
    for name in ("q", "k", "v", "out"):
        assert step(**{name: None}) == INVALID and step(**{name: FAKE + 8}) == INVALID
    assert step(workspace=None) == INVALID and step(workspace=FAKE + 64) == WORKSPACE and step(bytes=0) == WORKSPACE
    assert calls(lib, config(), tokens=-1, **bad)[0] == INVALID
    assert lib.adore_ring_fill(config(), FAKE, (1 << 24) + 1, rows(), rows(), None, FAKE, FAKE, None) == UNSUPPORTED
    for r in (None, rows(data=None), rows(data=FAKE + 4), rows(token=100), rows(head=-64)):
        assert lib.adore_ring_fill(config(), FAKE, 10, r, rows(), None, FAKE, FAKE, None) == INVALID
        assert lib.adore_ring_fill(config(), FAKE, 10, rows(), r, None, FAKE, FAKE, None) == INVALID
    assert lib.adore_ring_read(config(), FAKE, FAKE, None, FAKE, None) == INVALID and lib.adore_ring_read(config(), FAKE, FAKE, FAKE, FAKE + 8, None) == INVALID


def test_the_binding_refuses_what_does_not_fit():
    import torch
    from paper_2407_02328_amd import AdoreError, WindowCache
    how = dict(batch=1, heads=2, kv_heads=2, head_dim=64, dtype="bf16")
    with pytest.raises(AdoreError):
        WindowCache(window=0, **how)
    with pytest.raises(AdoreError):
        WindowCache(window=4, sinks=-1, **how)
    with pytest.raises(ValueError):
        WindowCache(window=4, scale=-1.0, **how)
    with pytest.raises(ValueError):
        WindowCache(window=4, cache=torch.zeros((1, 2, 1, 64 * 64), dtype=torch.bfloat16), **how)       # not on the GPU


def test_calls_take_place_on_the_device_of_their_tensors(monkeypatch):
    import torch
    from paper_2407_02328_amd import WindowCache, binding
    from tests.test_devices_cpu import Machine, OnGpu, on_gpu
    m, empty = Machine(), torch.empty
    monkeypatch.setattr(binding, "load_library", lambda: m)
    monkeypatch.setattr(binding, "_stream", lambda index: 0)
    monkeypatch.setattr(binding, "_current", lambda: m.current, raising=False)
    monkeypatch.setattr(torch.cuda, "device", m.device)
    monkeypatch.setattr(torch, "empty", lambda *args, device=None, **kw: empty(*args, **kw).as_subclass(OnGpu))
    cache, cursor = on_gpu((2 * 2 * 2 * 64 * 64 + 128,)), on_gpu((2, 2), torch.int32)
    at = -cache.data_ptr() % 256 // 2
    cache = cache[at:at + 2 * 2 * 2 * 64 * 64].view(2, 2, 2, 64 * 64)
    c = WindowCache(batch=2, heads=4, kv_heads=2, head_dim=64, window=60, sinks=4, dtype="bf16", cache=cache, cursor=cursor)
    c.fill(on_gpu((2, 2, 5, 64)), on_gpu((2, 2, 5, 64)), seen=on_gpu((2,), torch.int32))
    c.step(on_gpu((2, 4, 64)), on_gpu((2, 2, 64)), on_gpu((2, 2, 64)))
    c.read()
    assert m.calls == [("adore_ring_fill", 1), ("adore_ring_step", 1), ("adore_ring_read", 1)] and m.current == 0
    for bad in (lambda: c.fill(on_gpu((2, 2, 5, 64)), on_gpu((2, 2, 5, 64)), seen=on_gpu((3,), torch.int32)),
                lambda: c.fill(on_gpu((2, 2, 5, 64)), on_gpu((2, 2, 4, 64))), lambda: c.fill(on_gpu((2, 1, 5, 64)), on_gpu((2, 1, 5, 64))),
                lambda: c.step(on_gpu((2, 2, 64)), on_gpu((2, 2, 64)), on_gpu((2, 2, 64))),
                lambda: c.step(on_gpu((2, 4, 64), torch.float32), on_gpu((2, 2, 64)), on_gpu((2, 2, 64))),
                lambda: c.step(on_gpu((2, 64, 4)).transpose(1, 2), on_gpu((2, 2, 64)), on_gpu((2, 2, 64))), lambda: c.read(k=on_gpu((2, 2, 60, 64)))):
        with pytest.raises(ValueError):
            bad()
    assert len(m.calls) == 3
