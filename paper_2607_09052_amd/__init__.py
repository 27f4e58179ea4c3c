"""MI355X (gfx950) implementation of the COBS decode-step path.

The work happens in the HIP library libcobs.so (C ABI in include/cobs.h,
include/cobs_cache.h and include/cobs_tokens.h); ``cobs`` is its thin Python binding,
``cache`` that of the operators on the cache between decode steps, ``tokens`` that of
rotary positions, the append of new tokens and the 8-bit cache.
"""
from . import cache, cobs, tokens  # noqa: F401
