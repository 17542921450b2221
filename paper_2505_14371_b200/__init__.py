"""Layer-wise stochastic quantization + QODA update on one B200 (sm_100a), behind a C ABI.

`binding` marshals torch tensors into the C entry points of liblq.so (include/lq.h);
`rotary` makes the cache's tables of angles; `workloads` draws the seeded synthetic gradient sets; `build` compiles the library in-tree.
"""
from .binding import (CACHE_BAD_LENGTH, CACHE_BAD_PAGE, CACHE_BAD_POSITION, CACHE_BAD_SLOT, CACHE_NONFINITE, CODE_BROKEN, CODE_GAVE_UP, HIST_STRIDE, NUM_BINS, STATUS_NONFINITE, STATUS_ZERO_NORM, STEP_AUTO, Cache, LqError, Plan,
                      load_library, lq_code_build, lq_code_universal, lq_vector_norm_static)
from .rotary import lq_rotary_table

__all__ = ["Plan", "Cache", "lq_rotary_table", "CACHE_NONFINITE", "CACHE_BAD_SLOT", "CACHE_BAD_POSITION", "CACHE_BAD_PAGE", "CACHE_BAD_LENGTH",
           "LqError", "load_library", "lq_vector_norm_static", "lq_code_build", "lq_code_universal", "NUM_BINS", "HIST_STRIDE", "STATUS_ZERO_NORM",
           "STATUS_NONFINITE", "STEP_AUTO", "CODE_BROKEN", "CODE_GAVE_UP"]
