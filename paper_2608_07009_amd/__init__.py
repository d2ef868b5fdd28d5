"""HiSparse decode hot path on AMD Instinct MI355X (gfx950).

The compute lives in libhisparse.so (hand-written HIP kernels behind the C ABI of
include/hisparse.h); `hisparse` is its ctypes binding. `HiSparseCache` is a small convenience
owner of one handle.
"""
from .hisparse import (AttnDesc, CacheDesc, ChunkDesc, HisparseError, KvDesc,  # noqa: F401
                       hisparse_cache_create, hisparse_cache_destroy, hisparse_check_errors,
                       hisparse_chunk_attention, hisparse_chunk_workspace_bytes,
                       hisparse_decode_workspace_bytes, hisparse_fetch, hisparse_host_pool,
                       hisparse_kv_record_bytes, hisparse_layer_cache, hisparse_prefetch_layer,
                       hisparse_read_plan, hisparse_read_state, hisparse_read_tokens, hisparse_reset,
                       hisparse_resolve, hisparse_resolve_tables,
                       hisparse_sparse_decode, hisparse_sparse_decode_pool,
                       hisparse_status_string, hisparse_validate_attn, hisparse_validate_chunk,
                       hisparse_validate_desc, hisparse_validate_kv, hisparse_write_tokens,
                       host_view, lib)
from .cache import HiSparseCache  # noqa: F401
