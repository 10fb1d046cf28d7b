// Attention of the newest rows of every sequence over its paged cache, O = softmax(q K^T scale over the visible keys) V: the C entry points
// and how a call is cut into workgroups.
#include "cache_attn.h"

namespace veda {

// How a call is cut up.
struct AttnCut {
    int32_t size;       // rows of a block: 16 or 32 where a key head has no more rows than that for any sequence, else 128
    int32_t per_seq;    // see CacheAttnArgs
    int32_t workers;
    int32_t part_rows;
    int64_t items;
};
static AttnCut attn_cut(const veda_cache* c, const veda_cache_batch* b, int32_t q_heads, veda_visible vis) {
    AttnCut cut{};
    const int64_t max_new = b->max_new < b->rows ? b->max_new : b->rows, group = q_heads / c->kv_heads, rows = max_new * group;
    const bool bf16 = c->dtype == VEDA_BF16, few = rows <= 32;
    const int d = c->head_dim;
    cut.size = rows <= 16 ? 16 : rows <= 32 ? 32 : kAttnRows;
    // Even, so that the sums of a block, part_rows * (d + 2) floats, are whole 16 bytes: the list of cuts behind them is read 16 bytes at a time.
    cut.part_rows = few ? cut.size : rows < kAttnRows ? (int32_t)(rows + 1) & ~1 : kAttnRows;
    const int64_t each = (rows + cut.size - 1) / cut.size, uniform = b->seqs * each;
    cut.items = block_items(b->seqs, b->rows, max_new, group, cut.size);
    int64_t keys = (int64_t)b->max_pages * c->page_tokens;
    const bool countable = uniform <= 1024 && uniform * (keys / 16 + 8) < (int64_t)1 << 31;   // tiles; whatever the window, so that it never asks for more workspace
    if (vis.window) {   // what the rows of a block can see at most
        const int64_t span = (int64_t)vis.window + vis.sinks + (vis.block ? vis.block : 0) + kAttnRows;
        keys = keys < span ? keys : span;
    }
    // A batch is cut in one way, by the most rows that a sequence may have and the most keys that the table's width holds: a single token beside a
    // long prompt is a block of 128 rows (512 rows on 8192 keys and 63 ragged tokens 249 us, 98 and 186 apart; 4096 rows and a token on
    // 131,101 keys 2252 us, 135 and 105 apart: such are better two calls).
    // Shared out evenly where a block can have more keys than a workgroup's least part is worth and the blocks are too few to level out by
    // themselves: in a few rounds of workgroups the last one, or the longest, leaves compute units idle.  Every workgroup then counts
    // through all blocks, 64 at a time: up to 1024 of 16 or 32 rows, which are a sequence each, 256 of 128 rows.  Those are left as they are
    // where a workgroup for each fills four fifths of a round or comes in several rounds, and where a block's walk is not long against
    // what counting and joining take, 10-20 us and, in bf16, more the more blocks there are (d = 128, us without / with: 256 rows of 4 heads on
    // 456 keys 16 / 19, 756 21 / 20, 3756 72 / 23, 1024 rows of 12 heads, causal, on 1524 keys 38 / 40, 2524 56 / 44, 2133 rows of 12 on
    // 3633 keys 72 / 84, 1280 rows on 34,000 530 / 278-304 from box to box, 3840 872 / 734, 4680 985 / 1021; fp32, 100 rows of 12 on 160 keys 28 / 30, 200 38 / 30, 300 51 /
    // 30, 449 rows on 2000 302 / 63).
    const int64_t fit = few ? attn_keys_workers(bf16, c->head_dim) : attn_rows_workers(bf16), groups = uniform * c->kv_heads;
    // Few rows: long walks wait for memory, so eight waves a workgroup go through short caches about as fast as all that the card can hold, and
    // the joining is saved; in fp32, where products take longer, the more so the more workgroups there are (single tokens of 4 query heads a key
    // head, d = 128, us without / with: bf16, one cache of 6 heads, 700 keys 11 / 17, 2500 16 / 17, 4000 23 / 17; 32 ragged ones of 8 heads
    // up to 2500 27 / 36; 64, by two waves, up to 1000 28 / 33, 2500 68 / 63; fp32, one of 6 heads, 700 keys 20 / 24, 1500 35 / 24, 32 of 8 up to
    // 1500 42 / 47; d = 64, one of 6 heads 1500 21 / 23, 2500 30 / 23).
    const int64_t grown = (d == 64 ? 1536 : 768) + 8 * groups;
    const int64_t short_few = bf16 ? (groups <= 256 ? 2560 : 1536) : grown < 4096 ? grown : 4096;
    const bool share = keys > (few ? short_few : bf16 ? 512 + 16 * groups : 192) && countable &&
                       (few ? groups <= 8 * fit : uniform <= kRowsShareItems && 5 * groups < 4 * attn_rows_places());
    if (share) cut.workers = (int32_t)(fit < c->kv_heads ? c->kv_heads : fit / c->kv_heads * c->kv_heads);
    if (share || blocks_even(uniform, cut.items)) {
        cut.items = uniform;
        cut.per_seq = (int32_t)each;
    }
    return cut;
}
static size_t attn_workspace(const veda_cache* c, const AttnCut& cut) {
    if (!cut.workers) return 0;
    // unfinished sums with references and l: two blocks of few rows a workgroup, or the pieces of the others and how they were cut
    const size_t block = (size_t)cut.part_rows * (size_t)(c->head_dim + 2) * sizeof(float), groups = (size_t)cut.items * (size_t)c->kv_heads;
    return cut.size < kAttnRows ? (size_t)2 * cut.workers * block : ((size_t)2 * cut.workers + groups) * block + groups * 16;
}
static veda_status check_heads(const veda_cache* c, int32_t q_heads) {
    if (q_heads < 1 || q_heads % c->kv_heads) return VEDA_ERR_INVALID_ARG;
    return q_heads / c->kv_heads > 32 ? VEDA_ERR_UNSUPPORTED : VEDA_OK;
}

}  // namespace veda

extern "C" size_t veda_cache_attn_workspace_bytes(const veda_cache* c, const veda_cache_batch* b, int32_t q_heads) {
    if (veda::check_cache(c) != VEDA_OK || veda::check_batch(c, b) != VEDA_OK || veda::check_heads(c, q_heads) != VEDA_OK) return 0;
    return veda::attn_workspace(c, veda::attn_cut(c, b, q_heads, veda_visible{0, 0, 0}));
}

extern "C" veda_status veda_cache_attn_fwd(const veda_cache* c, const veda_cache_batch* b, int32_t q_heads, const void* q, veda_strides sq,
                                           float softmax_scale, veda_visible vis, void* out, veda_strides so, float* lse,
                                           void* workspace, size_t workspace_bytes, void* stream) {
    veda_status st = veda::check_cache(c);
    if (st == VEDA_OK) st = veda::check_batch(c, b);
    if (st == VEDA_OK) st = veda::check_heads(c, q_heads);
    if (st != VEDA_OK) return st;
    if (!(softmax_scale > 0.0f) || !(softmax_scale < INFINITY)) return VEDA_ERR_INVALID_ARG;
    constexpr int32_t kMost = 1 << 30;
    if (vis.block < 0 || vis.window < 0 || vis.sinks < 0 || vis.block > kMost || vis.window > kMost || vis.sinks > kMost) return VEDA_ERR_INVALID_ARG;
    if (b->seqs == 0 || b->rows == 0 || b->max_new == 0) return VEDA_OK;
    st = veda::check_rows(c, b->rows, q_heads, q, sq, false);
    if (st == VEDA_OK) st = veda::check_rows(c, b->rows, q_heads, out, so, true);
    if (st != VEDA_OK) return st;
    if (q == out) return VEDA_ERR_INVALID_ARG;   // a row may be read after its result has been written
    const veda::AttnCut cut = veda::attn_cut(c, b, q_heads, vis);
    const size_t need = veda::attn_workspace(c, cut);
    if (need > 0) {
        if (!workspace) return VEDA_ERR_INVALID_ARG;
        if (workspace_bytes < need) return VEDA_ERR_WORKSPACE;
        if (!veda::aligned16(workspace)) return VEDA_ERR_UNSUPPORTED;
    }
    const int es = c->dtype == VEDA_BF16 ? 2 : 4;
    veda::CacheAttnArgs a;
    a.c = veda::cache_args(c, b);
    a.q = (const char*)q; a.out = (char*)out; a.lse = lse;
    a.sq_h = sq.h * es; a.sq_n = sq.n * es; a.so_h = so.h * es; a.so_n = so.n * es;
    a.q_heads = q_heads; a.group = q_heads / c->kv_heads;
    a.items = cut.items; a.per_seq = cut.per_seq; a.workers = cut.workers; a.part_rows = cut.part_rows;
    a.block = vis.block; a.window = vis.window; a.sinks = vis.window ? vis.sinks : 0;
    a.scale_log2 = softmax_scale * veda::kLog2e;
    a.part = (float*)workspace;
    const bool bf16 = c->dtype == VEDA_BF16;
    // a grid has less than 2^32 threads: 512 to a workgroup, or to eight rows of a query head
    if (cut.items * c->kv_heads >= (int64_t)1 << 23 || (int64_t)a.c.max_new * a.group >= (int64_t)1 << 30 ||
        (cut.workers && cut.size < veda::kAttnRows && (int64_t)b->rows * q_heads >= (int64_t)1 << 26))
        return VEDA_ERR_UNSUPPORTED;
    const hipStream_t s = (hipStream_t)stream;
    return cut.size < veda::kAttnRows ? veda::launch_cache_attn_keys(a, bf16, c->head_dim, s) : veda::launch_cache_attn_rows(a, bf16, c->head_dim, s);
}
