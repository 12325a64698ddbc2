"""RBS-Attention sparse prefill on MI355X (gfx950): HIP kernels behind a C ABI.

    stats = rbs_block_stats(shape, K)                                  # Sec. 3.1
    rbs_stats_summarize(shape, stats)   # select-ready summary from centroids/radii/beta held elsewhere
    counts, indices = rbs_select(shape, Q, stats, tau_b, tau_r, sink, local, recent)  # Sec. 3.2
    O = rbs_sparse_prefill(shape, Q, K, V, counts, indices)            # Sec. 3.3
    counts, indices, O = rbs_select_attend(shape, Q, K, V, stats, ...)   # Sec. 3.2-3.3 in one call
    box = rbs_block_box(shape, K); rbs_select_variant(shape, Q, stats, "box", rho, ..., box=box)  # supporting selectors
    batch = Batch([n0, n1, ...]); shape = varlen_shape(batch, H_q, H_kv, B)   # independent sequences, packed
    stats = rbs_block_stats_varlen(shape, batch, K); ...; rbs_sparse_prefill_varlen(shape, batch, Q, K, V, ...)
    f8 = rbs_fp8_prepare(shape, Q, K, V); O = rbs_sparse_prefill_fp8(shape, f8, counts, indices)  # FP8 inputs

and around a paged key-value cache (the tokens that follow a prompt):

    pages = Pages.allocate(n_rows, max_pages, n_pages, page_size); cache = PagedCache.allocate(n_pages, page_size, H_kv)  # fp4=True: 4 bits
    step = rbs_pages_extend(pages, new_tokens, max_tokens)             # pages, positions, slots of new tokens
    Q, K = rbs_qk_norm_rope(shape, rope, Q, K, step.positions, V=V, cache=cache, slots=step.slots)
    O = rbs_paged_decode(shape, Q, cache, pages.page_table, step.seq_lens, cu_tokens=step.cu_tokens)
    O = rbs_paged_prefill(shape, Q, cache, pages.page_table, step.seq_lens, step.cu_tokens)  # all new tokens of each row
    rbs_cache_write(shape, K, V, cache, slots); K, V = rbs_cache_read(shape, cache, page_table, cu_tokens)  # plain rows
    rbs_pages_release(pages, released)                                 # finished rows
"""

from ._lib import (  # noqa: F401
    AUTO,
    attention_workspace,
    Fp8Inputs,
    allocate_fp8,
    rbs_fp8_amax,
    rbs_fp8_pack,
    rbs_fp8_prepare,
    rbs_fp8_vt_bytes,
    rbs_sparse_prefill_fp8,
    Batch,
    RBS_MAX_SEQS,
    allocate_lists_varlen,
    allocate_stats_varlen,
    rbs_batch,
    rbs_block_stats_varlen,
    rbs_dense_indices_varlen,
    rbs_select_varlen,
    rbs_sparse_prefill_varlen,
    rbs_varlen_blocks,
    rbs_varlen_index_capacity,
    rbs_varlen_summary_bytes,
    varlen_shape,
    BlockStats,
    BoxStats,
    SELECTORS,
    rbs_block_box,
    rbs_box,
    rbs_select_variant,
    RbsError,
    allocate_lists,
    load,
    make_shape,
    n_blocks,
    rbs_block_stats,
    rbs_stats_summarize,
    rbs_dense_indices,
    rbs_index_capacity,
    rbs_select,
    rbs_select_attend,
    rbs_shape,
    rbs_sparse_prefill,
    rbs_sparse_prefill_noalloc,
    rbs_stats,
    rbs_set_debug,
    rbs_status_str,
    rbs_summary_bytes,
    LIB_PATH,
    RBS_ERR_RANGE,
)
from ._paged import (  # noqa: F401
    RBS_CACHE_BF16,
    RBS_CACHE_FP4,
    RBS_CACHE_FP8,
    RBS_MAX_ROWS,
    RBS_PAGES_FEW,
    RBS_PAGES_ROW,
    RBS_PAGES_STACK,
    RBS_PAGES_TOKENS,
    PagedCache,
    Pages,
    PageStep,
    Rope,
    rbs_cache,
    rbs_cache_read,
    rbs_cache_write,
    rbs_decode_workspace_bytes,
    rbs_paged_decode,
    rbs_paged_prefill,
    rbs_pages,
    rbs_pages_extend,
    rbs_pages_release,
    rbs_prefill_workspace_bytes,
    rbs_qk_norm_rope,
    rbs_rope,
    rope_frequencies,
)
