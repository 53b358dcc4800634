"""Host-side checks of the rotation: its table of turns against exact arithmetic, and arguments that are refused before anything is
enqueued (the pointers are never dereferenced)."""
import ctypes
import math
from fractions import Fraction

import pytest

from paper_2407_02328_amd.binding import AdoreRotateConfig, Rotary
from tests.test_prompt_cpu import FAKE, INVALID, OK, UNSUPPORTED, WORKSPACE, lib, rows  # noqa: F401

GOOD = dict(batch=2, heads=4, kv_heads=2, head_dim=64, tokens=0, dtype=1, rotary_dim=64, interleaved=0, magnitude=1.0, eps=1e-6)
# 2 pi to 40 digits
TWO_PI = Fraction(62831853071795864769252867665590057683943, 10 ** 40)


def calls(lib, cfg, turns=FAKE, positions=FAKE, seq=0, token=1, qw=None, kw=None, **other):  # noqa: F811
    c = None if cfg is None else ctypes.byref(AdoreRotateConfig(**dict(GOOD, **cfg)))
    r = lambda name: other.get(name, rows())  # noqa: E731
    head = (c, turns, positions, seq, token, qw, kw)
    dqw, dkw = other.get("dqw", qw and FAKE), other.get("dkw", kw and FAKE)
    return (lib.adore_rotate_heads(*head, r("q"), r("k"), r("q_out"), r("k_out"), None),
            lib.adore_rotate_heads_backward(*head, r("d_q"), r("d_k"), r("q"), r("k"), r("dq"), r("dk"), dqw, dkw, other.get("workspace", FAKE),
                                            other.get("bytes", 1 << 24), None))


def test_nothing_to_do_is_fine(lib):  # noqa: F811
    assert calls(lib, {}) == (OK, OK)
    assert calls(lib, dict(kv_heads=0), k=None, k_out=None, d_k=None, dk=None) == (OK, OK)
    assert calls(lib, dict(rotary_dim=0), turns=None, positions=None) == (OK, OK)
    assert calls(lib, {}, qw=FAKE)[0] == OK


@pytest.mark.parametrize("change,code", [
    (dict(batch=0), INVALID), (dict(heads=0), INVALID), (dict(kv_heads=-1), INVALID), (dict(tokens=-1), INVALID), (dict(dtype=2), INVALID),
    (dict(head_dim=0), INVALID), (dict(rotary_dim=-16), INVALID), (dict(rotary_dim=80), INVALID), (dict(magnitude=-1.0), INVALID),
    (dict(magnitude=math.inf), INVALID), (dict(eps=-1e-6), INVALID), (dict(eps=math.nan), INVALID), (dict(head_dim=96), UNSUPPORTED),
    (dict(rotary_dim=24), UNSUPPORTED), (dict(tokens=(1 << 24) + 1), UNSUPPORTED), (dict(heads=8192), UNSUPPORTED), (dict(kv_heads=8192), UNSUPPORTED),
    (dict(batch=1 << 17), UNSUPPORTED)])
def test_configurations_are_refused(lib, change, code):  # noqa: F811
    assert calls(lib, change) == (code, code)
    assert lib.adore_rotate_backward_workspace_bytes(ctypes.byref(AdoreRotateConfig(**dict(GOOD, **change)))) == 0


def test_missing_and_misplaced_tensors_are_refused(lib):  # noqa: F811
    assert calls(lib, None) == (INVALID, INVALID)
    for kw in (dict(turns=None), dict(positions=None), dict(turns=FAKE + 4), dict(positions=FAKE + 2), dict(seq=-1), dict(token=-1), dict(qw=FAKE + 8),
               dict(kw=FAKE + 8)):
        assert calls(lib, {}, **kw) == (INVALID, INVALID), kw
    assert calls(lib, dict(kv_heads=0), k=None, k_out=None, d_k=None, dk=None, kw=FAKE) == (INVALID, INVALID)
    for bad in (None, rows(data=None), rows(data=FAKE + 8), rows(token=4), rows(head=-64), rows(seq=4), rows(token=(1 << 22) + 8)):
        for name in ("q_out", "k_out"):
            assert calls(lib, {}, **{name: bad})[0] == INVALID
        for name in ("d_q", "d_k", "dq", "dk"):
            assert calls(lib, {}, **{name: bad})[1] == INVALID
        assert calls(lib, {}, q=bad)[0] == calls(lib, {}, k=bad)[0] == INVALID
        assert calls(lib, {}, qw=FAKE, q=bad)[1] == calls(lib, {}, kw=FAKE, k=bad)[1] == INVALID
    assert calls(lib, dict(kv_heads=0))[0] == INVALID                       # a k that nobody counts
    for kw in (dict(qw=FAKE, dqw=None), dict(kw=FAKE, dkw=None), dict(dqw=FAKE), dict(dkw=FAKE)):
        assert calls(lib, {}, **kw)[1] == INVALID
    for kw in (dict(workspace=None), dict(workspace=FAKE + 16), dict(bytes=16)):
        assert calls(lib, {}, qw=FAKE, **kw)[1] == WORKSPACE


def test_workspace(lib):  # noqa: F811
    size = lambda **kw: lib.adore_rotate_backward_workspace_bytes(ctypes.byref(AdoreRotateConfig(**dict(GOOD, **kw))))  # noqa: E731
    assert size() >= 2 * 64 * 4
    assert size(tokens=1 << 20) == size(tokens=1 << 24) <= 512 * 2 * 64 * 4 + 256        # as many sums as there are places
    assert lib.adore_rotate_backward_workspace_bytes(None) == 0


@pytest.mark.parametrize("R,base,factor,original,low,high", [
    (128, 10000.0, 1.0, None, 1.0, 32.0), (64, 500000.0, 1.0, None, 1.0, 32.0), (32, 10000.0, 4.0, None, 1.0, 32.0), (128, 10000.0, 8.0, 4096.0, 1.0, 32.0),
    (96, 1e6, 32.0, 8192.0, 1.0, 4.0), (16, 0.01, 1.0, None, 1.0, 32.0)])
def test_turns(R, base, factor, original, low, high):
    """Frequencies as 2^64ths of a turn.  The roots and the blend here are Python's, within some 2^-52 of a frequency; the library's
    in 64 bits of mantissa: 2^-50 of a frequency, and half of a unit."""
    rotary = Rotary(R, base=base, factor=factor, original=original, low=low, high=high)
    assert rotary.turns.shape == (R // 2,)
    for j, got in enumerate(int(t) % (1 << 64) for t in rotary.turns):
        f = base ** (-2.0 * j / R)
        whole = 0.0 if original is None else min(max((original * f / (2 * math.pi) - low) / (high - low), 0.0), 1.0)
        f *= whole + (1.0 - whole) / factor
        exact = Fraction(f) / TWO_PI * 2 ** 64
        off = (Fraction(got) - exact) % 2 ** 64
        off = min(off, 2 ** 64 - off)
        assert off <= exact / 2 ** 50 + 1, (j, float(off))


def test_turns_of_powers_are_exact(lib):  # noqa: F811
    """base = 2^k with whole exponents: the frequency is a power of two, and its turns are 2^64 / 2 pi shifted."""
    turns = (ctypes.c_uint64 * 8)()
    assert lib.adore_rotary_turns(16, 2.0 ** 16, 1.0, 0.0, 1.0, 32.0, turns) == OK
    for j in range(8):                              # f = 2^(-2 j)
        assert abs(turns[j] - Fraction(1, 4 ** j) / TWO_PI * 2 ** 64) <= 1


def test_tables_are_refused(lib):  # noqa: F811
    turns = (ctypes.c_uint64 * 32)()
    for args in ((0, 1e4, 1.0, 0.0, 1.0, 32.0), (7, 1e4, 1.0, 0.0, 1.0, 32.0), (64, 0.0, 1.0, 0.0, 1.0, 32.0), (64, -1.0, 1.0, 0.0, 1.0, 32.0),
                 (64, math.inf, 1.0, 0.0, 1.0, 32.0), (64, 1e4, 0.0, 0.0, 1.0, 32.0), (64, 1e4, math.nan, 0.0, 1.0, 32.0), (64, 1e4, 1.0, -1.0, 1.0, 32.0),
                 (64, 1e4, 2.0, 4096.0, 32.0, 1.0), (64, 1e4, 2.0, 4096.0, math.nan, 1.0), (64, 1e-30, 1.0, 0.0, 1.0, 32.0)):
        assert lib.adore_rotary_turns(*args, turns) == INVALID, args
    assert lib.adore_rotary_turns(64, 1e4, 1.0, 0.0, 1.0, 32.0, None) == INVALID


def test_the_binding_refuses_what_does_not_fit():
    import torch
    from paper_2407_02328_amd import AdoreError, rotate_heads
    for kw in (dict(rotary_dim=24), dict(rotary_dim=0), dict(rotary_dim=64, magnitude=0.0), dict(rotary_dim=64, original=0.0)):
        with pytest.raises(ValueError):
            Rotary(**kw)
    with pytest.raises(AdoreError):
        Rotary(64, base=-1.0)
    q = torch.zeros((4, 2, 64), dtype=torch.bfloat16)
    with pytest.raises(ValueError):
        rotate_heads(q, None, torch.zeros(4, dtype=torch.int32), Rotary(64))       # not on the GPU


class TestShapes:
    """What the binding holds tensors to, with tensors that say they are on a device."""

    @pytest.fixture
    def machine(self, monkeypatch):
        import torch
        from paper_2407_02328_amd import binding
        from tests.test_devices_cpu import Machine, OnGpu
        m, empty = Machine(), torch.empty
        m.adore_rotary_turns = lambda *a: 0
        monkeypatch.setattr(binding, "load_library", lambda: m)
        monkeypatch.setattr(binding, "_stream", lambda index: 0)
        monkeypatch.setattr(binding, "_current", lambda: m.current, raising=False)
        monkeypatch.setattr(torch.cuda, "device", m.device)
        strided = torch.empty_strided
        monkeypatch.setattr(torch, "empty", lambda *args, device=None, **kw: empty(*args, **kw).as_subclass(OnGpu))
        monkeypatch.setattr(torch, "empty_strided", lambda *args, device=None, **kw: strided(*args, **kw).as_subclass(OnGpu))
        return m

    def test_on_their_device_and_to_q_s_shape(self, machine, monkeypatch):
        import torch
        from paper_2407_02328_amd import rotate_heads, rotate_heads_backward
        from tests.test_devices_cpu import on_gpu
        rotary = Rotary(64)
        monkeypatch.setattr(Rotary, "on", lambda self, device: FAKE)
        q, k, pos = on_gpu((5, 4, 64)), on_gpu((5, 2, 64)), on_gpu((5,), torch.int32)
        w = on_gpu((64,), torch.float32)
        rotate_heads(q, k, pos, rotary, q_weight=w)
        rotate_heads_backward(q, k, q, k, pos, rotary, q_weight=w)
        assert [c for c in machine.calls if c[0] != "adore_rotary_turns"] == [("adore_rotate_heads", 1), ("adore_rotate_heads_backward", 1)]
        assert machine.current == 0
        dense, dk = on_gpu((2, 4, 5, 64)), on_gpu((2, 2, 5, 64))
        rotate_heads(dense, dk, on_gpu((2, 5), torch.int32), rotary)
        rotate_heads(dense, dk, pos, rotary)
        n = len(machine.calls)
        for args, kw in (((q, on_gpu((4, 2, 64)), pos, rotary), {}), ((q, on_gpu((5, 2, 128)), pos, rotary), {}), ((q, dk, pos, rotary), {}),
                         ((q, k, on_gpu((4,), torch.int32), rotary), {}), ((q, k, on_gpu((5,), torch.int64), rotary), {}), ((q, k, None, rotary), {}),
                         ((q, k, on_gpu((1,), torch.int32), rotary), {}), ((dense, dk, on_gpu((1, 5), torch.int32), rotary), {}),
                         ((q, k, pos, None), {}), ((q, k, pos, rotary), dict(q_weight=on_gpu((64,)))), ((q, k, pos, rotary), dict(q_weight=on_gpu((32,), torch.float32))),
                         ((q, None, pos, rotary), dict(k_weight=w)), ((q, k, pos, rotary), dict(eps=-1.0)), ((q, k, pos, rotary), dict(q_out=k)),
                         ((q, None, pos, rotary), dict(k_out=k)), ((q, k, pos, rotary), dict(k_out=on_gpu((1, 2, 64)).expand(5, 2, 64))),
                         ((on_gpu((5, 64)), None, pos, rotary), {}), ((q, on_gpu((5, 2, 64), torch.float32), pos, rotary), {}),
                         ((on_gpu((5, 4, 32)), None, pos, rotary), {})):
            with pytest.raises(ValueError):
                rotate_heads(*args, **kw)
        with pytest.raises(ValueError):
            rotate_heads_backward(q, k, q, None, pos, rotary)
        assert len(machine.calls) == n
