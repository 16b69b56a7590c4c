"""MI355X (gfx950) MOD-DiT hot path: mask predictor + block-sparse attention.

The compute lives in libmoddit.so (HIP kernels behind the C ABI declared in
include/moddit.h); this package only binds it.
"""
from ._capi import *  # noqa: F401,F403
from ._capi import (EXPORTED, LIB_PATH, Cache, ModError, Rope, Stats, make_budget,  # noqa: F401
                    make_cache, make_cache_shape, make_params, make_rope_params, make_shape, raw_lib)
