"""MI355X-native EVA attention (FlashEVA's fused window + summary attention).

The compute lives in libeva.so (hand-written HIP for gfx950 behind the C ABI
in include/eva.h); `eva` is the torch-facing binding, `inputs` the seeded
synthetic workloads.  Importing the package does not load the library; the
first call does, and raises if it is not built.
"""
from .eva import (Cache, PagedCache, PageTable, QuantCache, RaggedCache, append_path, build_summaries,  # noqa: F401
                  cache_append, cache_fill, decode_step, page_extend, page_truncate, paged_append, paged_decode,
                  paged_select, prefill, prefill_attention, qappend_decode, qcache_append, qcache_fill, qcache_read,
                  qdecode_step, qk_norm_rope, qk_norm_rope_backward, rope_turns, tree_attention)
