"""MI355X-native implementation of ADORE's per-step decode path (arXiv 2407.02328).

`binding.Adore` wraps the C-ABI library libadore.so (HIP kernels for gfx950);
`build.build_library()` compiles it in-tree.
"""
from .binding import (Adore, AdoreConfig, AdoreError, EXPORTS, EXPORTS_Q4, KERNELS, LIB_PATH, Q4Cache, load_library,  # noqa: F401
                      make_config, prompt_attention, prompt_attention_backward, prompt_scores, topk_attention)
