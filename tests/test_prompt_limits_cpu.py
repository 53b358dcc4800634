"""The largest problems of the calls on prompts: what is taken can be launched, fewer than 2^32 threads."""
import ctypes

import pytest

from paper_2407_02328_amd.binding import AdorePromptConfig
from tests.test_prompt_cpu import GOOD, lib  # noqa: F401


@pytest.mark.parametrize("change,packed,taken", [
    # 2^24 blocks of 32 tokens x heads, and 2^24 workgroups of 128 tokens too
    (dict(batch=1 << 16, heads=256, kv_heads=256, q_tokens=32, k_tokens=32), 0, False),
    (dict(batch=1 << 16, heads=256, kv_heads=256, q_tokens=1, k_tokens=1), 0, False),
    (dict(batch=1 << 16, heads=256, kv_heads=1, q_tokens=0, k_tokens=32), 0, False),
    (dict(batch=(1 << 16) - 1, heads=256, kv_heads=256, q_tokens=32, k_tokens=32), 0, True),
    (dict(batch=1 << 16, heads=255, kv_heads=255, q_tokens=32, k_tokens=32), 0, True),
    (dict(batch=1, heads=4096, kv_heads=4096, q_tokens=1 << 17, k_tokens=1 << 17), 0, False),
    (dict(batch=1, heads=4096, kv_heads=4096, q_tokens=(1 << 17) - 32, k_tokens=(1 << 17) - 32), 0, True),
    # packed: a block more for every sequence, and one
    (dict(batch=1, heads=4096, kv_heads=4096, q_tokens=32 * 4094, k_tokens=0), 1, False),
    (dict(batch=1, heads=4096, kv_heads=4096, q_tokens=32 * 4093, k_tokens=0), 1, True),
])
def test_how_many_workgroups(lib, change, packed, taken):  # noqa: F811
    cfg = AdorePromptConfig(**dict(GOOD, **change))
    assert (lib.adore_prompt_backward_workspace_bytes(ctypes.byref(cfg), packed) > 0) == taken
    rows = 128
    for n, heads in ((cfg.q_tokens, cfg.heads), (cfg.k_tokens, cfg.kv_heads)):
        blocks = n // rows + cfg.batch + 1 if packed else cfg.batch * -(-n // rows)
        assert not taken or blocks * heads * 256 < 1 << 32
