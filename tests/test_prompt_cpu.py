"""Host-side checks of the calls on whole prompts: arguments are refused before anything is enqueued (the pointers used here are
never dereferenced)."""
import ctypes
import os

import pytest

from paper_2407_02328_amd import LIB_PATH, load_library
from paper_2407_02328_amd.binding import AdorePromptConfig, AdoreRows

FAKE = 0x7F0000000000
OK, INVALID, UNSUPPORTED, WORKSPACE = 0, -1, -3, -4
GOOD = dict(batch=2, heads=4, kv_heads=2, head_dim=64, q_tokens=0, k_tokens=0, dtype=1, scale=0.0)


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(LIB_PATH):
        from paper_2407_02328_amd.build import build_library
        build_library()
    return load_library()


def rows(**kw):
    return ctypes.byref(AdoreRows(**dict(dict(data=FAKE, seq=0, token=256, head=64), **kw)))


def calls(lib, cfg, q_start=FAKE, k_start=FAKE, **other):
    """Return codes of the three calls with q_tokens = k_tokens = 0, which enqueue nothing; other: tensors by name."""
    r = lambda name: other.get(name, rows())  # noqa: E731
    c = None if cfg is None else ctypes.byref(cfg)
    lse, ws = other.get("lse", FAKE), other.get("workspace", FAKE)
    return (lib.adore_prompt_attention(c, q_start, k_start, r("q"), r("k"), r("v"), r("out"), lse, other.get("rest"), None),
            lib.adore_prompt_attention_backward(c, q_start, k_start, r("d_out"), r("q"), r("k"), r("v"), r("out"), other.get("rest"), lse, r("dq"),
                                                r("dk"), r("dv"), ws, other.get("bytes", 1 << 20), None),
            lib.adore_prompt_scores(c, q_start, k_start, r("q"), r("k"), lse, other.get("scores", FAKE), None))


def test_nothing_to_do_is_fine(lib):
    assert calls(lib, AdorePromptConfig(**GOOD))[::2] == (OK, OK)


@pytest.mark.parametrize("change,code", [
    (dict(batch=0), INVALID), (dict(heads=0), INVALID), (dict(kv_heads=3), INVALID), (dict(kv_heads=0), INVALID), (dict(q_tokens=-1), INVALID),
    (dict(k_tokens=-1), INVALID), (dict(dtype=2), INVALID), (dict(scale=-1.0), INVALID), (dict(scale=float("nan")), INVALID),
    (dict(scale=float("inf")), INVALID), (dict(head_dim=0), INVALID), (dict(head_dim=96), UNSUPPORTED), (dict(q_tokens=(1 << 24) + 1), UNSUPPORTED),
    (dict(heads=8192, kv_heads=8192), UNSUPPORTED), (dict(batch=1 << 17), UNSUPPORTED), (dict(heads=4096, q_tokens=1 << 22), UNSUPPORTED)])
def test_configurations_are_refused(lib, change, code):
    cfg = AdorePromptConfig(**dict(GOOD, **change))
    assert calls(lib, cfg) == (code, code, code)
    assert lib.adore_prompt_backward_workspace_bytes(ctypes.byref(cfg), 1) == 0


def test_missing_and_misplaced_tensors_are_refused(lib):
    cfg = AdorePromptConfig(**GOOD)
    assert calls(lib, None) == (INVALID,) * 3
    assert calls(lib, cfg, q_start=None) == (INVALID,) * 3
    assert calls(lib, cfg, k_start=None) == (INVALID,) * 3
    for bad in (None, rows(data=None), rows(data=FAKE + 8), rows(token=4), rows(head=-64), rows(seq=4), rows(token=(1 << 22) + 8)):
        assert calls(lib, cfg, q=bad) == (INVALID,) * 3
        assert calls(lib, cfg, k=bad) == (INVALID,) * 3
        assert calls(lib, cfg, v=bad)[:2] == (INVALID,) * 2
        assert calls(lib, cfg, out=bad)[:2] == (INVALID,) * 2
        for name in ("d_out", "dq", "dk", "dv"):
            assert calls(lib, cfg, **{name: bad})[1] == INVALID
    assert calls(lib, cfg, lse=None)[1:] == (INVALID,) * 2
    assert calls(lib, cfg, scores=None)[2] == INVALID
    assert calls(lib, cfg, workspace=None)[1] == INVALID
    assert calls(lib, cfg, workspace=FAKE + 16)[1] == WORKSPACE
    assert calls(lib, cfg, bytes=0)[1] == WORKSPACE
    f32 = AdorePromptConfig(**dict(GOOD, dtype=0))
    assert calls(lib, f32, rest=rows())[:2] == (INVALID,) * 2      # nothing is lost in fp32
    assert calls(lib, cfg, rest=rows(data=FAKE + 2))[:2] == (INVALID,) * 2


def test_workspace_of_the_backward_pass(lib):
    cfg = AdorePromptConfig(**dict(GOOD, q_tokens=1000, k_tokens=1000))
    size = lib.adore_prompt_backward_workspace_bytes
    assert 4 * 4 * 1000 <= size(ctypes.byref(cfg), 1) < size(ctypes.byref(cfg), 0)
    assert size(ctypes.byref(cfg), 0) >= 2 * 4 * 4 * 1000 and size(ctypes.byref(cfg), 0) % 256 == 0
    assert size(None, 1) == 0


def test_the_binding_refuses_tensors_that_do_not_fit():
    import torch
    from paper_2407_02328_amd import prompt_attention
    q = torch.zeros((4, 2, 64), dtype=torch.bfloat16)
    with pytest.raises(ValueError):
        prompt_attention(q, q, q)                       # not on the GPU
    with pytest.raises(ValueError):
        prompt_attention(q, q, q, q_start=torch.zeros(2, dtype=torch.int32))
