"""MI355X-native balanced block-sparse attention (the single-GPU hot path of db-SP, arXiv 2511.23113).

The product is libdbsp.so (HIP for gfx950 + a C++ host planner) behind the C ABI declared in
include/dbsp.h; this package is its thin Python binding.
"""

from .binding import (  # noqa: F401
    DBSP_EHIP,
    DBSP_EINVAL,
    DBSP_ENOMEM,
    DBSP_ESHAPE,
    DBSP_OK,
    DbspError,
    HeadNorm,
    KVCache,
    MODE_BALANCED,
    MODE_NAIVE,
    MODE_REWARD,
    MODE_ROUNDS,
    PagedKVCache,
    Plan,
    Rotary,
    cache_attn_fwd,
    cache_evict,
    fit_cost_model,
    imbalance_ratio,
    load_library,
    mfma_probe,
    paged_append,
    paged_attn_fwd,
    partition_blocks,
    partition_heads,
    plan_sparse_attn,
    plan_sparse_attn_reuse,
    qk_norm_rope_bwd,
    qk_norm_rope_fwd,
    ring_work,
    sparse_attn_fwd,
)
