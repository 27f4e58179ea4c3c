"""MI355X (gfx950) implementation of the COBS decode-step path.

The work happens in the HIP library libcobs.so (C ABI in include/cobs.h and
include/cobs_cache.h); ``cobs`` is its thin Python binding, ``cache`` that of
the operators on the cache between decode steps.
"""
from . import cache, cobs  # noqa: F401
