"""MI355X-native capture-and-stage path for model-internal observability.

The product is libdmi.so (HIP kernels + C ABI, see include/dmi.h); this package
only marshals arguments for it.
"""
from .binding import (DmiError, KV8, KV8Batch, PreparedBatch, PreparedObserve, Ring, Step, Stats, RecordView,  # noqa: F401
                      kv8_append, kv8_attend, kv8_attend_workspace, kv8_evict, lib, library_path, record_bytes, version)
from . import binding  # noqa: F401
