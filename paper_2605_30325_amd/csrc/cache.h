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
// A tensor of rows [rows][heads][head_dim] in the caller's memory: aligned, strides of 16 bytes, and (distinct) no two rows with a byte in common.
// An axis of one entry has no stride, whatever it is given as: s.n or s.h becomes 0.
veda_status check_rows(const veda_cache* c, int32_t rows, int32_t heads, const void* p, veda_strides& s, bool distinct);

// Copies pages of `bytes` (a multiple of 16) inside both pools; see veda_cache_copy_pages.
veda_status copy_pages(char* k, char* v, int64_t page_b, int64_t bytes, int32_t pages, const int32_t* pairs, int64_t n, hipStream_t s, const char* what);

#if defined(__HIPCC__)

// Sum over the lanes up to and with this one, by DPP; all 64 lanes take part.
__device__ __forceinline__ int lanes_up_to(int x) {
    x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xf, 0xf, false);   // row_shr:1, 2, 4, 8
    x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xf, 0xf, false);
    x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xf, 0xf, false);
    x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xf, 0xf, false);
    x += __builtin_amdgcn_update_dpp(0, x, 0x142, 0xa, 0xf, false);   // row_bcast:15, 31
    x += __builtin_amdgcn_update_dpp(0, x, 0x143, 0xc, 0xf, false);
    return x;
}

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

// Work items: every sequence's rows in blocks (of `size`, where a token counts as `group` rows), sequence by sequence.  Only the
// device knows the sequences' lengths; a grid of the longest's blocks for each of them is mostly empty where they are ragged, and an empty
// workgroup costs its launch: prompts of 4096 rows and less, 8192 workgroups of which 4168 empty, 527 us instead
// of 352 with the items numbered as here.  Returns false for numbers beyond the last item.
struct RowBlock { int seq, block, blocks; SeqRows rows; };   // block of blocks of its sequence
__device__ __forceinline__ bool find_block(const CacheArgs& c, int group, int size, int item, RowBlock& out) {
    const int lane = threadIdx.x & 63;
    int base = 0;
    for (int s0 = 0; s0 < c.seqs; s0 += 64) {
        SeqRows r{0, 0, 0};
        if (s0 + lane < c.seqs) r = seq_rows(c, s0 + lane);
        const int blocks = (int)(((int64_t)min(r.n, c.max_new) * group + size - 1) / size);
        const int up_to = lanes_up_to(blocks);
        const int total = __builtin_amdgcn_readlane(up_to, 63);
        if (item < base + total) {
            const int at = __popcll(__ballot(base + up_to <= item));
            out.seq = s0 + at;
            out.blocks = __builtin_amdgcn_readlane(blocks, at);
            out.block = item - (base + __builtin_amdgcn_readlane(up_to, at) - out.blocks);
            out.rows = SeqRows{__builtin_amdgcn_readlane(r.first, at), __builtin_amdgcn_readlane(r.n, at), __builtin_amdgcn_readlane(r.len, at)};
            return true;
        }
        base += total;
    }
    return false;
}
// Item -> block of rows: by division where the grid has per_seq for every sequence, else (0) by what the sequences hold.
__device__ __forceinline__ bool block_of(const CacheArgs& c, int group, int size, int per_seq, int item, RowBlock& out) {
    if (!per_seq) return find_block(c, group, size, item, out);
    out.seq = item / per_seq;
    out.block = item % per_seq;
    out.rows = seq_rows(c, out.seq);
    out.blocks = (int)(((int64_t)min(out.rows.n, c.max_new) * group + size - 1) / size);
    return out.block < out.blocks;
}
// Items that a grid has to have, as far as the host knows.
inline int64_t block_items(int64_t seqs, int64_t rows, int64_t max_new, int64_t group, int64_t size) {
    const int64_t each = seqs * ((max_new * group + size - 1) / size), all = rows * group / size + seqs;
    return each < all ? each : all;
}
// Whether few of `uniform` blocks, the longest sequence's for each, can be empty, so that there is no need to search for those that are not.
inline bool blocks_even(int64_t uniform, int64_t items) { return uniform <= items + items / 4; }

#endif

}  // namespace veda
