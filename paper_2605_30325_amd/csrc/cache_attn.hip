// Attention of the newest rows of every sequence over its paged cache, O = softmax(q K^T scale over the visible keys) V: the C entry points
// and how a call is cut into workgroups.
#include "cache_attn.h"
#include "packed.h"

namespace veda {

// Keys up to which few rows of a packed cache are left to a workgroup for each block and key head: eight waves up to 256 of them, four up to 768, two
// beyond, as many as run at once.  The waves of a workgroup go through their tiles one after the other, and the longest cache of a batch decides; sharing levels
// lengths out, but takes 17 to 21 us however short the walk, most of it looking up and joining.  Single tokens of 4 query heads a key head, lengths of any size up to
// the one given, us apart / shared: bf16, d = 128, one cache of 6 heads, 2000 keys 17 / 19, 3000 22 / 19; 32 of 8, 3000 24 / 28, 5000 34 / 32, 7000 44 / 36; 64 of 8, 2000 28 /
// 30, 3000 37 / 35, 4500 52 / 41; 128 of 8, 1200 29 / 36, 2000 47 / 44, 3000 67 / 56; 512 of 8, 3800 237 / 270; d = 64, one of 6, 2500 16 / 17, 3000 17 / 17; 32 of 8,
// 5000 26 / 29, 7000 32 / 31; 64 of 8, 3000 28 / 28, 4500 39 / 32; 128 of 8, 2000 36 / 34; fp32, d = 128, one of 6, 2000 20 / 21, 3000 27 / 21; 32 of 8, 3000 29 / 31, 4500 38 /
// 34; 64 of 8, 2000 33 / 33, 4500 63 / 47; 512 of 8, 3000 240 / 243, 3800 309 / 302; d = 64, 32 of 8, 7000 38 / 33; 64 of 8, 3000 32 / 30.
// Caches of one length have nothing to level out, and are up to a fifth faster apart beyond the threshold too (bf16, d = 128, 64 of 8, 3000 40 / 45, 96 of 8, 2800 57 / 68;
// fp32, 64 of 8, 2000 36 / 40), but lengths are on the device.  Blocks of 17 to 32 rows go by the same thresholds, which are those of single tokens (8 tokens of 4 query heads,
// d = 128: bf16, 64 of 8, 2000 39 / 52, 3000 51 / 59, 128 of 8, 2000 70 / 85; fp32, whose short walk spills registers, 16 of 8, 2000 56 / 44, 3000 76 / 40, 64 of 8, 2000 99 / 66).
static int64_t packed_short(bool bf16, int d, int64_t groups) {
    if (groups <= 256) return d == 64 ? 2700 + 20 * groups : bf16 ? 2400 + 10 * groups : 2200 + 8 * groups;
    if (groups <= 768) return d == 64 ? 3600 : bf16 ? 2800 : 2000;
    return (d == 64 || bf16 ? 1400 : 1000) + groups * 3 / 5;
}

// How a call is cut up.
struct AttnCut {
    int32_t size;       // rows of a block: 16 or 32 where a key head has no more rows than that for any sequence, else 128 or 256
    int32_t per_seq;    // see CacheAttnArgs
    int32_t workers;
    int32_t part_rows;
    int64_t items;
    size_t bytes;       // of workspace
};
// unfinished sums with references and l: two blocks of few rows a workgroup, or the pieces of the others and how they were cut
static size_t attn_workspace(const veda_cache* c, const AttnCut& cut) {
    if (!cut.workers) return 0;
    const size_t block = (size_t)cut.part_rows * (size_t)(c->head_dim + 2) * sizeof(float), groups = (size_t)cut.items * (size_t)c->kv_heads;
    return cut.size < kAttnRows ? (size_t)2 * cut.workers * block : ((size_t)2 * cut.workers + groups) * block + groups * 16;
}
static AttnCut attn_cut(const veda_cache* c, bool packed, const veda_cache_batch* b, int32_t q_heads, veda_visible vis) {
    AttnCut cut{};
    const int64_t max_new = b->max_new < b->rows ? b->max_new : b->rows, group = q_heads / c->kv_heads, rows = max_new * group;
    const bool bf16 = c->dtype == VEDA_BF16, few = rows <= 32;
    const int d = c->head_dim;
    cut.size = rows <= 16 ? 16 : rows <= 32 ? 32 : kAttnRows;
    // Even, so that the sums of a block, part_rows * (d + 2) floats, are whole 16 bytes: the list of cuts behind them is read 16 bytes at a time.
    cut.part_rows = few ? cut.size : rows < kAttnRows ? (int32_t)(rows + 1) & ~1 : kAttnRows;
    int64_t each = (rows + cut.size - 1) / cut.size, uniform = b->seqs * each;
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
    // fp32 rows of a packed cache: at d = 64 two workgroups fit a compute unit, which pays where they have five tiles each at least (12 heads on 4 key
    // heads, us with 512 / 256: 449 rows of two sequences on 8449 keys 91 / 102, on 2449 43 / 43, 333 rows on 2033 34 / 33; 2464 rows of 12 heads, causal,
    // on 4464 106 / 129).
    const bool many = bf16 || (packed && d == 64 && uniform * c->kv_heads * (keys / 64) >= 5 * attn_rows_workers(true));
    const int64_t fit = !few ? attn_rows_workers(many) : packed ? packed_keys_workers(bf16, d, cut.size) : attn_keys_workers(bf16, d), groups = uniform * c->kv_heads;
    // Few rows: long walks wait for memory, so eight waves a workgroup go through short caches about as fast as all that the card can hold, and
    // the joining is saved; in fp32, where products take longer, the more so the more workgroups there are (single tokens of 4 query heads a key
    // head, d = 128, us without / with: bf16, one cache of 6 heads, 700 keys 11 / 17, 2500 16 / 17, 4000 23 / 17; 32 ragged ones of 8 heads
    // up to 2500 27 / 36; 64, by two waves, up to 1000 28 / 33, 2500 68 / 63; fp32, one of 6 heads, 700 keys 20 / 24, 1500 35 / 24, 32 of 8 up to
    // 1500 42 / 47; d = 64, one of 6 heads 1500 21 / 23, 2500 30 / 23).
    const int64_t grown = (d == 64 ? 1536 : 768) + 8 * groups;
    const int64_t short_few = packed ? packed_short(bf16, d, groups) : bf16 ? (groups <= 256 ? 2560 : 1536) : grown < 4096 ? grown : 4096;
    const bool share = keys > (few ? short_few : bf16 ? 512 + 16 * groups : 192) && countable &&
                       (few ? groups <= 8 * fit : uniform <= kRowsShareItems && 5 * groups < 4 * attn_rows_places());
    // bf16 rows of a packed cache, d = 128: blocks of 256 rows, whose eight waves turn a tile's codes into values once where two blocks of 128 do it
    // twice, but load, begin and end together.  Where that fills no more than a quarter of rows in vain, and walks are long: of two tiles at least
    // for each workgroup that shares, of 4096 keys in several rounds of workgroups, 10240 in one (causal, or frames of 1560, us with 128 / 256: 12 heads, 4680 rows on
    // 36,240 keys 1036 / 918, 12,680 385 / 363, 8680 242 / 254, 3840 rows on 35,840 888 / 801, 640 on 32,640 161 / 153, 300 on 32,300 100 / 106, 130 on 3130 30 / 27,
    // 256 on 1256 29 / 31; 8 sequences of 512 rows of 32 heads on 8, 4512 keys 289 / 271, 512 44 / 46).  d = 64, where a tile has half as much to turn: never (4680 rows
    // on 8680 keys 170 / 186).
    auto finish = [&](int64_t at_once) {
        if (share) cut.workers = (int32_t)(at_once < c->kv_heads ? c->kv_heads : at_once / c->kv_heads * c->kv_heads);
        if (share || blocks_even(uniform, cut.items)) {
            cut.items = uniform;
            cut.per_seq = (int32_t)each;
        }
        const size_t bytes = attn_workspace(c, cut);
        cut.bytes = bytes > cut.bytes ? bytes : cut.bytes;      // of either way: a window that leaves blocks of 128 must not ask for more than none did
    };
    finish(fit);
    const int64_t tall = (rows + 2 * kAttnRows - 1) / (2 * kAttnRows);
    if (packed && bf16 && d == 128 && rows > kAttnRows && 8 * tall <= 5 * each &&
        (share ? b->seqs * tall * c->kv_heads * (keys / 64) >= fit : keys >= (groups >= 1024 ? 4096 : 10240) && 5 * groups >= 4 * attn_rows_places())) {
        cut.size = cut.part_rows = 2 * kAttnRows;
        cut.per_seq = 0;
        each = tall;
        uniform = b->seqs * each;
        cut.items = block_items(b->seqs, b->rows, max_new, group, cut.size);
        finish(fit / 2);
    }
    return cut;
}
static veda_status check_heads(const veda_cache* c, int32_t q_heads) {
    if (q_heads < 1 || q_heads % c->kv_heads) return VEDA_ERR_INVALID_ARG;
    return q_heads / c->kv_heads > 32 ? VEDA_ERR_UNSUPPORTED : VEDA_OK;
}

// Workspace of a call on a cache of these rows (c), checked already.
static size_t attn_bytes(const veda_cache* c, bool packed, const veda_cache_batch* b, int32_t q_heads) {
    if (check_batch(c, b) != VEDA_OK || check_heads(c, q_heads) != VEDA_OK) return 0;
    return attn_cut(c, packed, b, q_heads, veda_visible{0, 0, 0}).bytes;
}
// The call on a cache of these rows, checked already; pools: what its kernels see.
static veda_status attend(const veda_cache* c, const CacheArgs& pools, bool packed, const veda_cache_batch* b, int32_t q_heads, const void* q, veda_strides sq,
                          float softmax_scale, veda_visible vis, void* out, veda_strides so, float* lse, void* workspace, size_t workspace_bytes,
                          hipStream_t s) {
    veda_status st = check_heads(c, q_heads);
    if (st != VEDA_OK) return st;
    if (!(softmax_scale > 0.0f) || !(softmax_scale < INFINITY)) return VEDA_ERR_INVALID_ARG;
    constexpr int32_t kMost = 1 << 30;
    if (vis.block < 0 || vis.window < 0 || vis.sinks < 0 || vis.block > kMost || vis.window > kMost || vis.sinks > kMost) return VEDA_ERR_INVALID_ARG;
    if (b->seqs == 0 || b->rows == 0 || b->max_new == 0) return VEDA_OK;
    st = check_rows(c, b->rows, q_heads, q, sq, false);
    if (st == VEDA_OK) st = check_rows(c, b->rows, q_heads, out, so, true);
    if (st != VEDA_OK) return st;
    if (q == out) return VEDA_ERR_INVALID_ARG;   // a row may be read after its result has been written
    const AttnCut cut = attn_cut(c, packed, b, q_heads, vis);
    if (cut.bytes > 0) {
        if (!workspace) return VEDA_ERR_INVALID_ARG;
        if (workspace_bytes < cut.bytes) return VEDA_ERR_WORKSPACE;
        if (!aligned16(workspace)) return VEDA_ERR_UNSUPPORTED;
    }
    const int es = c->dtype == VEDA_BF16 ? 2 : 4;
    CacheAttnArgs a;
    a.c = pools;
    a.q = (const char*)q; a.out = (char*)out; a.lse = lse;
    a.sq_h = sq.h * es; a.sq_n = sq.n * es; a.so_h = so.h * es; a.so_n = so.n * es;
    a.q_heads = q_heads; a.group = q_heads / c->kv_heads;
    a.items = cut.items; a.per_seq = cut.per_seq; a.workers = cut.workers; a.part_rows = cut.part_rows;
    a.block = vis.block; a.window = vis.window; a.sinks = vis.window ? vis.sinks : 0;
    a.scale_log2 = softmax_scale * kLog2e;
    a.part = (float*)workspace;
    const bool bf16 = c->dtype == VEDA_BF16;
    // a grid has less than 2^32 threads: 512 to a workgroup, or to eight rows of a query head
    if (cut.items * c->kv_heads >= (int64_t)1 << 23 || (int64_t)a.c.max_new * a.group >= (int64_t)1 << 30 ||
        (cut.workers && cut.size < kAttnRows && (int64_t)b->rows * q_heads >= (int64_t)1 << 26))
        return VEDA_ERR_UNSUPPORTED;
    if (packed) return cut.size < kAttnRows ? launch_packed_attn_keys(a, bf16, c->head_dim, s) : launch_packed_attn_rows(a, bf16, c->head_dim, s);
    return cut.size < kAttnRows ? launch_cache_attn_keys(a, bf16, c->head_dim, s) : launch_cache_attn_rows(a, bf16, c->head_dim, s);
}

}  // namespace veda

extern "C" size_t veda_cache_attn_workspace_bytes(const veda_cache* c, const veda_cache_batch* b, int32_t q_heads) {
    return veda::check_cache(c) == VEDA_OK ? veda::attn_bytes(c, false, b, q_heads) : 0;
}

extern "C" veda_status veda_cache_attn_fwd(const veda_cache* c, const veda_cache_batch* b, int32_t q_heads, const void* q, veda_strides sq,
                                           float softmax_scale, veda_visible vis, void* out, veda_strides so, float* lse,
                                           void* workspace, size_t workspace_bytes, void* stream) {
    veda_status st = veda::check_cache(c);
    if (st == VEDA_OK) st = veda::check_batch(c, b);
    if (st != VEDA_OK) return st;
    return veda::attend(c, veda::cache_args(c, b), false, b, q_heads, q, sq, softmax_scale, vis, out, so, lse, workspace, workspace_bytes,
                        (hipStream_t)stream);
}

extern "C" size_t veda_packed_attn_workspace_bytes(const veda_packed_cache* c, const veda_cache_batch* b, int32_t q_heads) {
    if (veda::check_packed(c) != VEDA_OK) return 0;
    const veda_cache as = veda::packed_rows(c);
    return veda::attn_bytes(&as, true, b, q_heads);
}

extern "C" veda_status veda_packed_attn_fwd(const veda_packed_cache* c, const veda_cache_batch* b, int32_t q_heads, const void* q, veda_strides sq,
                                            float softmax_scale, veda_visible vis, void* out, veda_strides so, float* lse,
                                            void* workspace, size_t workspace_bytes, void* stream) {
    veda_status st = veda::check_packed(c);
    if (st != VEDA_OK) return st;
    const veda_cache as = veda::packed_rows(c);
    st = veda::check_batch(&as, b);
    if (st != VEDA_OK) return st;
    return veda::attend(&as, veda::packed_args(c, b), true, b, q_heads, q, sq, softmax_scale, vis, out, so, lse, workspace, workspace_bytes,
                        (hipStream_t)stream);
}
