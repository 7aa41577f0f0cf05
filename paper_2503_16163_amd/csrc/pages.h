// What the calls on a paged cache share: its checks, and what a kernel reads it by.
#pragma once
#include "operators.h"

namespace specache {

constexpr int64_t kMostPositions = 1ll << 28;

struct PageArgs {
    specache_view k, v, bounds;       // (a view's batch stride goes from page to page)
    const int32_t* table;
    int64_t table_stride;
    int n_pages, n_kv_heads, log2, table_pages;
};

inline int check_pages(const specache_pages* c) {
    if (!c) return fail_without_context(SPECACHE_EINVAL, "null cache");
    if (c->head_dim != kD) return fail_without_context(SPECACHE_EINVAL, "head_dim must be 128");
    if (c->dtype != SPECACHE_FP16 && c->dtype != SPECACHE_BF16) return fail_without_context(SPECACHE_EINVAL, "dtype must be SPECACHE_FP16 or SPECACHE_BF16");
    if (c->n_pages < 0 || c->n_kv_heads < 1 || c->n_kv_heads > (1 << 20) || c->table_pages < 0 || c->table_stride < 0)
        return fail_without_context(SPECACHE_EINVAL, "n_pages, table_pages and table_stride must not be negative, n_kv_heads positive");
    if (c->page_tokens < 16 || c->page_tokens > 256 || (c->page_tokens & (c->page_tokens - 1)))
        return fail_without_context(SPECACHE_EINVAL, "page_tokens must be 16, 32, 64, 128 or 256");
    if ((int64_t)c->table_pages * c->page_tokens > kMostPositions) return fail_without_context(SPECACHE_EINVAL, "too many positions in the table");
    return SPECACHE_OK;
}
// the memory behind it, where a call reaches for it
inline int check_page_views(const specache_pages& c, bool pairs, bool bounds) {
    if (c.table_pages && (!c.table || (uintptr_t)c.table % 4)) return fail_without_context(SPECACHE_EINVAL, "null or misaligned table");
    if (!c.n_pages) return SPECACHE_OK;
    if ((pairs && (!view_fits(c.k) || !view_fits(c.v))) || (bounds && !view_fits(c.bounds)))
        return fail_without_context(SPECACHE_EINVAL, "a view's address must be 16-byte aligned, its strides multiples of 8");
    if (pairs && (c.k.token > (1 << 20) || c.v.token > (1 << 20))) return fail_without_context(SPECACHE_EINVAL, "strides from place to place go up to 2^20");
    return SPECACHE_OK;
}
inline PageArgs page_args(const specache_pages& c) {
    return PageArgs{c.k, c.v, c.bounds, c.table, c.table_stride, c.n_pages, c.n_kv_heads, __builtin_ctz((unsigned)c.page_tokens), c.table_pages};
}

// checks of a block call, and what specache_block_attend needs of scratch memory
int check_blocks(const specache_pages* cache, const specache_block_config* c);
int block_attend_scratch(const specache_pages& cache, const specache_block_config& c, int64_t* bytes);

}  // namespace specache
