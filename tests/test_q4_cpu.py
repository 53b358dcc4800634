"""Host-side checks of the calls on the cache held in 4 bits: sizes, and arguments that are refused before anything is enqueued."""
import ctypes
import os
import re

import pytest

from paper_2407_02328_amd import EXPORTS_Q4, LIB_PATH, load_library
from paper_2407_02328_amd.binding import AdoreQ4Config, AdoreRows

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
FAKE = 0x7F0000000000
INVALID, UNSUPPORTED, WORKSPACE = -1, -3, -4
GOOD = dict(batch=2, heads=4, kv_heads=2, head_dim=64, slots=100, recent=5, dtype=1, scale=0.0)


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(LIB_PATH):
        from paper_2407_02328_amd.build import build_library
        build_library()
    return load_library()


def test_symbols_of_the_header_are_exported(lib):
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "adore.h")).read(), flags=re.S)
    declared = set(re.findall(r"\b(adore_q4_[a-z]+(?:_[a-z]+)*)\s*\(", text))
    assert declared == set(EXPORTS_Q4)
    for name in declared:
        assert hasattr(lib, name)


def config(**kw):
    return ctypes.byref(AdoreQ4Config(**dict(GOOD, **kw)))


def test_sizes(lib):
    assert lib.adore_q4_cache_bytes(config()) == 2 * 2 * 2 * 68 * 64
    assert lib.adore_q4_cache_bytes(config(slots=64)) == 2 * 2 * 1 * 68 * 64
    assert lib.adore_q4_cache_bytes(config(slots=65, head_dim=128)) == 2 * 2 * 2 * 68 * 128
    for kw in ({}, dict(slots=20000), dict(heads=48, kv_heads=1), dict(batch=512), dict(heads=32, kv_heads=2, slots=4096, batch=300)):
        assert lib.adore_q4_workspace_bytes(config(**kw)) >= 256
    # a long cache's exponents, one per query head and slot, go through the workspace
    assert lib.adore_q4_workspace_bytes(config(slots=20000)) >= 2 * 4 * 20000 * 4
    assert lib.adore_q4_cache_bytes(None) == 0 and lib.adore_q4_workspace_bytes(None) == 0


REFUSED = [(dict(batch=0), INVALID), (dict(heads=3), INVALID), (dict(kv_heads=0), INVALID), (dict(slots=1, recent=1), INVALID), (dict(recent=0), INVALID),
           (dict(recent=100), INVALID), (dict(dtype=3), INVALID), (dict(scale=-0.5), INVALID), (dict(scale=float("inf")), INVALID), (dict(head_dim=0), INVALID),
           (dict(head_dim=80), UNSUPPORTED), (dict(slots=(1 << 20) + 1), UNSUPPORTED), (dict(batch=1 << 17), UNSUPPORTED), (dict(heads=8192), UNSUPPORTED),
           (dict(batch=1024, slots=1 << 20), UNSUPPORTED)]


def calls(lib, cfg, **other):
    p = lambda name: other.get(name, FAKE)  # noqa: E731
    r = lambda name: other.get(name, ctypes.byref(AdoreRows(FAKE, 0, 128, 64)))  # noqa: E731
    state = [p(n) for n in ("cache", "slot_pos", "score", "cursor")]
    return (lib.adore_q4_fill(cfg, p("k_start"), other.get("tokens", 10), r("k_rows"), r("v_rows"), p("scores"), *state, None),
            lib.adore_q4_step(cfg, p("q"), p("k"), p("v"), *state, p("out"), p("k_held"), p("v_held"), p("workspace"), other.get("bytes", 1 << 30), None),
            lib.adore_q4_read(cfg, state[0], state[1], p("k"), p("v"), None))


@pytest.mark.parametrize("change,code", REFUSED)
def test_configurations_are_refused(lib, change, code):
    assert calls(lib, config(**change)) == (code,) * 3
    assert lib.adore_q4_cache_bytes(config(**change)) == 0 and lib.adore_q4_workspace_bytes(config(**change)) == 0


def test_missing_and_misplaced_buffers_are_refused(lib):
    # every call below has something that is refused: none enqueues
    bad_cfg = None
    assert calls(lib, bad_cfg) == (INVALID,) * 3
    for name, off in (("cache", 128), ("slot_pos", 4)):
        for value in (None, FAKE + off):
            assert calls(lib, config(), **{name: value}) == (INVALID,) * 3
    state_only = dict(cache=FAKE + 128)             # (keeps the calls that a change does not concern from enqueuing)
    for name, off in (("score", 4), ("cursor", 4)):
        for value in (None, FAKE + off):
            assert calls(lib, config(), **dict(state_only, **{name: value}))[:2] == (INVALID,) * 2
    lib_step = lambda **kw: lib.adore_q4_step(config(), *[kw.get(n, FAKE) for n in ("q", "k", "v", "cache", "slot_pos", "score", "cursor", "out", "k_held", "v_held", "workspace")],  # noqa: E731
                                              kw.get("bytes", 1 << 30), None)
    for name in ("q", "k", "v", "out"):
        assert lib_step(**{name: None}) == INVALID and lib_step(**{name: FAKE + 8}) == INVALID
    for name in ("score", "cursor"):
        assert lib_step(**{name: None}) == INVALID and lib_step(**{name: FAKE + 4}) == INVALID
    assert lib_step(k_held=FAKE + 2) == INVALID and lib_step(v_held=FAKE + 2) == INVALID
    assert lib_step(workspace=None) == INVALID and lib_step(workspace=FAKE + 64) == WORKSPACE and lib_step(bytes=0) == WORKSPACE
    lib_fill = lambda **kw: lib.adore_q4_fill(config(), kw.get("k_start", FAKE), kw.get("tokens", 10), kw.get("k", ctypes.byref(AdoreRows(FAKE, 0, 128, 64))),  # noqa: E731
                                              kw.get("v", ctypes.byref(AdoreRows(FAKE, 0, 128, 64))), FAKE, FAKE, FAKE, kw.get("score", FAKE), kw.get("cursor", FAKE), None)
    assert lib_fill(tokens=-1) == INVALID and lib_fill(tokens=(1 << 24) + 1) == UNSUPPORTED
    for rows in (None, ctypes.byref(AdoreRows(None, 0, 128, 64)), ctypes.byref(AdoreRows(FAKE + 4, 0, 128, 64)), ctypes.byref(AdoreRows(FAKE, 0, 100, 64)),
                 ctypes.byref(AdoreRows(FAKE, 0, 128, -64))):
        assert lib_fill(k=rows) == INVALID and lib_fill(v=rows) == INVALID
    assert lib_fill(score=None) == INVALID and lib_fill(cursor=None) == INVALID
    assert lib.adore_q4_read(config(), FAKE, FAKE, None, FAKE, None) == INVALID and lib.adore_q4_read(config(), FAKE, FAKE, FAKE, FAKE + 8, None) == INVALID


def test_the_binding_refuses_what_does_not_fit():
    import torch
    from paper_2407_02328_amd import AdoreError, Q4Cache
    with pytest.raises(AdoreError):
        Q4Cache(batch=1, heads=2, kv_heads=2, head_dim=64, slots=8, recent=8, dtype="bf16")
    with pytest.raises(ValueError):
        Q4Cache(batch=1, heads=2, kv_heads=2, head_dim=64, slots=8, recent=1, dtype="bf16", scale=-1.0)
    with pytest.raises(ValueError):
        Q4Cache(batch=1, heads=2, kv_heads=2, head_dim=64, slots=8, recent=1, dtype="bf16", cache=torch.zeros((1, 2, 1, 68 * 64), dtype=torch.uint8))
