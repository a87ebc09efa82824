"""MI355X-native decode attention over a block-wise low-rank KV cache.

The work runs in libmilo.so (hand-written gfx950 HIP kernels behind the C ABI
declared in include/milo.h); `milo` is a thin ctypes binding with the same
entry-point names.  Besides the decode / prefill attention it holds the
encoder's entropy rank allocation (milo_allocate_ranks) and the paged 8-bit cache
of the requests' own keys and values (milo_pages_*, milo_attend_pages).
"""
from . import milo  # noqa: F401
from .milo import (MILO_KV_E4M3, MILO_KV_INT8, MiloError, MiloPages, lib, milo_allocate_ranks,  # noqa: F401
                   milo_attend_decode, milo_attend_pages, milo_attend_prefill, milo_cache_create,
                   milo_cache_device_bytes, milo_cache_free, milo_cache_read_factor, milo_last_error, milo_pages_create,
                   milo_pages_load, milo_pages_plan, milo_pages_store, milo_timing_enable, milo_timing_read,
                   milo_timing_read_alloc)
