"""vecattn: vertical-vector sparse attention for AMD MI355X (gfx950).

After VecAttention (arXiv 2603.29494): per query block, pool the queries
(Eq. 2), score every key with the pooled query and keep the important key
columns (row-wise topK budget, topP mass threshold, or the minS filter of
Eq. 3, also with Algorithm 1's cross-tile running maximum; Sec. 3.1), then run
attention restricted to the gathered K/V rows of those columns (Eq. 4,
Algorithm 2).  Beside them: attention with a sliding window and sinks, and for
the tokens after the prompt a paged key/value cache held in 4 or 8 bits and
attention over it.  All of it is HIP kernels in libvecattn.so behind the C ABI
of include/vecattn.h; this package only marshals torch tensors to it.
"""
from ._lib import (SEL_MINS, SEL_MINS_TILED, SEL_TOPK, SEL_TOPP, Cache, VecattnError, attn_order,
                   cache_alloc, cache_attn, cache_attn_workspace_bytes, cache_bytes, cache_read,
                   cache_write, check_lists,
                   head_sparsity, head_sparsity_of, load, max_count, plan_filter_ratios, pool,
                   recall, select, select_varlen, sparse_attn, sparse_attn_varlen, varlen_blocks,
                   window_attn, workspace_bytes)

__all__ = ["SEL_TOPK", "SEL_TOPP", "SEL_MINS", "SEL_MINS_TILED", "Cache", "VecattnError",
           "attn_order", "cache_alloc", "cache_attn", "cache_attn_workspace_bytes", "cache_bytes",
           "cache_read", "cache_write", "check_lists",
           "head_sparsity", "head_sparsity_of", "recall",
           "load", "max_count", "plan_filter_ratios", "pool", "select", "select_varlen",
           "sparse_attn", "sparse_attn_varlen", "varlen_blocks", "window_attn", "workspace_bytes"]
