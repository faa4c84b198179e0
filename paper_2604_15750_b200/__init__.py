"""DepCap block-step on B200: Python binding over the C-ABI CUDA library (libdepcap.so).

Argument marshalling only; every step of the path runs in the library's kernels.
"""
from .binding import (DepCap, DepCapError, Hyper, lib, load_library, pack_kv_cache,  # noqa: F401
                      STAGE_NAMES, signals_static)
from .ops import (KvCache, cache_read, cache_write, qk_norm_rope, tree_attention,  # noqa: F401
                  tree_attention_workspace, tree_mask)
