"""Host-side checks of attention with a window: arguments are refused before anything is enqueued (the pointers are never dereferenced)."""
import ctypes

import pytest

from paper_2407_02328_amd.binding import AdorePromptConfig, AdoreWindow, _window
from tests.test_prompt_cpu import FAKE, GOOD, INVALID, OK, WORKSPACE, lib, rows  # noqa: F401

BIG = dict(GOOD, q_tokens=5000, k_tokens=5000)


def window(w, s):
    return ctypes.byref(AdoreWindow(w, s))


def calls(lib, cfg, win, starts=(FAKE, FAKE), space=FAKE, size=1 << 20):  # noqa: F811
    c, r = ctypes.byref(AdorePromptConfig(**cfg)), rows()
    return (lib.adore_window_attention(c, win, *starts, r, r, r, r, FAKE, None, None),
            lib.adore_window_attention_backward(c, win, *starts, r, r, r, r, r, None, FAKE, r, r, r, space, size, None))


def test_nothing_to_do_is_fine(lib):  # noqa: F811
    assert calls(lib, GOOD, window(1, 0)) == (OK, OK)


@pytest.mark.parametrize("w,s", [(0, 0), (-1, 0), (1, -1), (0, 5)])
def test_windows_are_refused(lib, w, s):  # noqa: F811
    assert calls(lib, GOOD, window(w, s)) == (INVALID, INVALID)
    assert lib.adore_window_backward_workspace_bytes(ctypes.byref(AdorePromptConfig(**GOOD)), window(w, s), 1) == 0


def test_what_plain_attention_refuses_is_refused(lib):  # noqa: F811
    assert calls(lib, GOOD, None) == (INVALID, INVALID)
    assert calls(lib, dict(GOOD, head_dim=96), window(4, 0)) == (-3, -3)
    assert calls(lib, GOOD, window(4, 0), starts=(FAKE, None)) == (INVALID, INVALID)
    assert calls(lib, GOOD, window(4, 0), space=FAKE + 16)[1] == WORKSPACE
    assert calls(lib, BIG, window(4, 0), size=4096)[1] == WORKSPACE


@pytest.mark.parametrize("packed", [0, 1])
def test_workspace(lib, packed):  # noqa: F811
    """What plain attention wants, and the first keys' sums where queries are cut: 32 keys x 2 x head_dim in fp32 a place."""
    cfg = ctypes.byref(AdorePromptConfig(**BIG))
    plain = lib.adore_prompt_backward_workspace_bytes(cfg, packed)
    size = lambda w, s: lib.adore_window_backward_workspace_bytes(cfg, window(w, s), packed)  # noqa: E731
    assert size(100, 0) == plain and size(5000, 4) == plain and size(1 << 30, 1 << 30) == plain
    assert size(100, 4) > plain and (size(100, 4) - plain) % (2 * 2 * 64 * 64 * 4) == 0
    assert (size(100, 65) - plain) % (2 * 4 * 64 * 64 * 4) == 0 and size(100, 65) > plain       # (another 64 keys a place)


def test_places_of_chunks_lie_in_the_workspace(lib):  # noqa: F811
    """The places that the kernels work out from starts, whatever those hold, against the bytes that were asked for."""
    import random
    rng = random.Random(3)
    for _ in range(300):
        batch, tokens, W = rng.randint(1, 40), rng.randint(600, 9000), rng.choice([1, 3, 50, 500, 3000])
        cfg = dict(GOOD, batch=batch, q_tokens=tokens, k_tokens=tokens)
        extra = lib.adore_window_backward_workspace_bytes(ctypes.byref(AdorePromptConfig(**cfg)), window(W, 4), 1) - \
            lib.adore_prompt_backward_workspace_bytes(ctypes.byref(AdorePromptConfig(**cfg)), 1)
        if extra == 0:
            continue
        slots = extra // (2 * 2 * 64 * 64 * 4)
        # the chunk is not handed out: 128 queries at these sizes
        chunk = 128
        sorted_starts = rng.random() < 0.7
        qs = [rng.randint(-5, tokens + 5) for _ in range(batch + 1)]
        ks = [rng.randint(-5, tokens + 5) for _ in range(batch + 1)]
        if sorted_starts:
            qs, ks = sorted(qs), sorted(ks)
        cut = lambda s: min(max(s, 0), tokens)  # noqa: E731
        taken = set()
        for b in range(batch):
            q0, k0 = cut(qs[b]), cut(ks[b])
            nq, nk = max(cut(qs[b + 1]) - q0, 0), max(cut(ks[b + 1]) - k0, 0)
            far = nq - max(W - (nk - nq), 0)           # queries as far as the window from the first key
            if far <= 0:
                continue
            assert nk > W
            first = q0 // chunk + min(b, k0 // (W + 1))
            mine = set(range(first, first + -(-far // chunk)))
            assert max(mine) < slots
            if sorted_starts:
                assert not mine & taken
            taken |= mine


def test_the_binding_refuses_what_does_not_fit():
    import torch
    from paper_2407_02328_amd import prompt_attention
    assert _window(None, 0) is None
    for w, s in ((0, 0), (-3, 0), (4, -1), (None, 2)):
        with pytest.raises(ValueError):
            _window(w, s)
    q = torch.zeros((4, 2, 64), dtype=torch.bfloat16)
    with pytest.raises(ValueError):
        prompt_attention(q, q, q, window=0)
