// The paged cache as the kernels see it, and the checks that its calls share.  Not part of the public ABI.
#pragma once

#include "veda_internal.h"

namespace veda {

struct CacheArgs {
    char *k, *v;
    int64_t page_b;                 // bytes from a page to the next
    int32_t pages, log_page, kv_heads;
    const int32_t *table, *kv_len, *q_start;
    int64_t table_stride;
    int32_t seqs, rows, max_new, max_pages;
};

veda_status check_cache(const veda_cache* c);
veda_status check_batch(const veda_cache* c, const veda_cache_batch* b);   // after check_cache
CacheArgs cache_args(const veda_cache* c, const veda_cache_batch* b);
// A tensor of rows [rows][heads][head_dim] in the caller's memory: aligned, strides of 16 bytes, and (distinct) no two rows the same bytes.
veda_status check_rows(const veda_cache* c, int32_t rows, int32_t heads, const void* p, veda_strides s, bool distinct);

#if defined(__HIPCC__)

// Rows and length of a sequence, whatever the arrays hold.
struct SeqRows {
    int first;    // row of its first new token
    int n;        // new tokens
    int len;      // tokens, the new ones among them
};
__device__ __forceinline__ SeqRows seq_rows(const CacheArgs& c, int s) {
    SeqRows r;
    r.first = min(max(c.q_start[s], 0), c.rows);
    r.n = max(min(c.q_start[s + 1], c.rows) - r.first, 0);
    r.len = min(max(c.kv_len[s], 0), c.max_pages << c.log_page);
    return r;
}

#endif

}  // namespace veda
