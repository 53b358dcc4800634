"""MI355X-native implementation of ADORE's per-step decode path (arXiv 2407.02328).

`binding.Adore` wraps the C-ABI library libadore.so (HIP kernels for gfx950);
`build.build_library()` compiles it in-tree.
"""
from .binding import (Adore, AdoreConfig, AdoreError, EXPORTS, EXPORTS_Q4, KERNELS, LIB_PATH, Q4Cache, Rotary, WindowCache,  # noqa: F401
                      load_library, make_config, prompt_attention, prompt_attention_backward, prompt_scores, rotate_heads,
                      rotate_heads_backward, topk_attention)
