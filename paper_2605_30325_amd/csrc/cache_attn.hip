// Attention of the newest rows of every sequence over its paged cache, O = softmax(q K^T scale over the visible keys) V: the C entry points,
// how a call is cut into workgroups, and the joining of split keys.
#include "cache_attn.h"

namespace veda {

// Puts the splits of a (row, query head) together, a workgroup for each: its waves take every fourth split, four loads in flight, and
// meet in LDS.  (One wave for all splits, one after the other: 36 us for 64 splits of 40 rows, most of it latency.)
template <bool kBf16, int D> __global__ __launch_bounds__(256) void cache_attn_join_splits_kernel(CacheAttnArgs a) {
    constexpr int C = D / 64;
    __shared__ float sums[4][D + 2];
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    const int64_t row = blockIdx.x, part_rows = (int64_t)a.c.rows * a.q_heads;
    const int token = (int)(row / a.q_heads), qh = (int)(row % a.q_heads);
    bool mine = false;   // is the row one of a sequence
    for (int s = lane; s < a.c.seqs; s += 64) {
        const int first = max(a.c.q_start[s], 0), last = a.c.q_start[s + 1];
        mine = mine || (token >= first && token < last && token - first < a.c.max_new);
    }
    if (!__any(mine)) return;
    const float2* ml = reinterpret_cast<const float2*>(a.part + a.splits * part_rows * D) + row;
    float ref = -INFINITY;
    for (int s = lane; s < a.splits; s += 64) ref = fmaxf(ref, ml[s * part_rows].x);
#pragma unroll
    for (int w = 32; w >= 1; w >>= 1) ref = fmaxf(ref, __shfl_xor(ref, w));
    float l = 0.0f, o[C];
#pragma unroll
    for (int c = 0; c < C; ++c) o[c] = 0.0f;
    for (int s0 = wave; s0 < a.splits; s0 += 16) {
        float2 m[4];
        float x[4][C];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int64_t at = (int64_t)min(s0 + 4 * j, a.splits - 1) * part_rows;
            m[j] = ml[at];
#pragma unroll
            for (int c = 0; c < C; ++c) x[j][c] = a.part[(at + row) * D + C * lane + c];
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            if (s0 + 4 * j >= a.splits || m[j].y == 0.0f) continue;   // a split without keys
            const float f = m[j].x == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(m[j].x - ref);   // -inf: the sum is NaN
            l += f * m[j].y;
#pragma unroll
            for (int c = 0; c < C; ++c) o[c] += f * x[j][c];
        }
    }
#pragma unroll
    for (int c = 0; c < C; ++c) sums[wave][C * lane + c] = o[c];
    if (lane == 0) sums[wave][D] = l;
    __syncthreads();
    if (wave != 0) return;
    l = sums[0][D] + sums[1][D] + sums[2][D] + sums[3][D];
    const float inv = attn_inverse(l);
    char* dst = a.out + token * a.so_n + (int64_t)qh * a.so_h;
#pragma unroll
    for (int c = 0; c < C; ++c) {
        const int ch = C * lane + c;
        const float y = (sums[0][ch] + sums[1][ch] + sums[2][ch] + sums[3][ch]) * inv;
        if constexpr (kBf16) reinterpret_cast<__bf16*>(dst)[ch] = (__bf16)y;
        else reinterpret_cast<float*>(dst)[ch] = y;
    }
    if (a.lse && lane == 0) a.lse[(int64_t)qh * a.c.rows + token] = attn_lse(ref, l);
}

// How a call is cut up.
struct AttnCut {
    int32_t few;        // 16 or 32: no more rows than that for a key head (cache_attn_keys.hip); 0: blocks of rows (cache_attn_rows.hip)
    int32_t per_seq;    // see CacheAttnArgs
    int32_t workers, splits;
    int64_t items;      // blocks of rows of one key head, at most
};
static AttnCut attn_cut(const veda_cache* c, const veda_cache_batch* b, int32_t q_heads, veda_visible vis) {
    AttnCut cut{0, 0, 0, 1, 0};
    const int64_t max_new = b->max_new < b->rows ? b->max_new : b->rows, group = q_heads / c->kv_heads, rows = max_new * group;
    const bool bf16 = c->dtype == VEDA_BF16;
    cut.few = rows <= 16 ? 16 : rows <= 32 ? 32 : 0;
    const int64_t size = cut.few ? cut.few : kAttnRows, each = (rows + size - 1) / size;
    cut.items = block_items(b->seqs, b->rows, max_new, group, size);
    if (b->seqs * each <= cut.items + cut.items / 4) {   // few of them can be empty: no search
        cut.items = b->seqs * each;
        cut.per_seq = (int32_t)each;
    }
    int64_t keys = (int64_t)b->max_pages * c->page_tokens;
    if (vis.window) {   // what the rows of a block can see at most
        const int64_t span = (int64_t)vis.window + vis.sinks + (vis.block ? vis.block : 0) + kAttnRows;
        keys = keys < span ? keys : span;
    }
    const int64_t items = cut.items * c->kv_heads;
    if (cut.few) {
        // Shared out evenly where some sequence can be longer than a workgroup's least part and the blocks of rows are too few to level
        // out by themselves; the sequences are counted through by every workgroup, 64 at a time.
        const int64_t fit = attn_keys_workers(bf16, c->head_dim);
        if (keys > 512 && items <= 8 * fit && b->seqs <= 1024 && b->seqs * (keys / 32 + 8) < (int64_t)1 << 31)
            cut.workers = (int32_t)(fit < c->kv_heads ? c->kv_heads : fit / c->kv_heads * c->kv_heads);
        return cut;
    }
    // Splits of the keys where the blocks of rows alone do not fill the compute units twice, of 512 keys or more.
    const int64_t most = (keys + 511) / 512;
    int64_t splits = items > 0 ? 512 / items : 1;
    if (splits > most) splits = most;
    cut.splits = splits < 1 ? 1 : (int32_t)splits;
    return cut;
}
static size_t attn_workspace(const veda_cache* c, const veda_cache_batch* b, int32_t q_heads, const AttnCut& cut) {
    const size_t row = (size_t)(c->head_dim + 2) * sizeof(float);
    if (cut.workers) return (size_t)2 * (size_t)cut.workers * (size_t)cut.few * row;
    return cut.splits < 2 ? 0 : (size_t)cut.splits * (size_t)b->rows * (size_t)q_heads * row;
}
static veda_status check_heads(const veda_cache* c, int32_t q_heads) {
    if (q_heads < 1 || q_heads % c->kv_heads) return VEDA_ERR_INVALID_ARG;
    return q_heads / c->kv_heads > 32 ? VEDA_ERR_UNSUPPORTED : VEDA_OK;
}

}  // namespace veda

extern "C" size_t veda_cache_attn_workspace_bytes(const veda_cache* c, const veda_cache_batch* b, int32_t q_heads) {
    if (veda::check_cache(c) != VEDA_OK || veda::check_batch(c, b) != VEDA_OK || veda::check_heads(c, q_heads) != VEDA_OK) return 0;
    return veda::attn_workspace(c, b, q_heads, veda::attn_cut(c, b, q_heads, veda_visible{0, 0, 0}));
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
    const veda::AttnCut cut = veda::attn_cut(c, b, q_heads, vis);
    const size_t need = veda::attn_workspace(c, b, q_heads, cut);
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
    a.splits = cut.splits; a.per_seq = cut.per_seq; a.workers = cut.workers;
    a.block = vis.block; a.window = vis.window; a.sinks = vis.window ? vis.sinks : 0;
    a.scale_log2 = softmax_scale * veda::kLog2e;
    a.part = (float*)workspace;
    const bool bf16 = c->dtype == VEDA_BF16;
    const int64_t groups = cut.workers ? cut.workers : cut.items * c->kv_heads * cut.splits;
    const bool joined = cut.workers || cut.splits > 1;
    if (groups >= (int64_t)1 << 31 || (int64_t)a.c.max_new * a.group >= (int64_t)1 << 30 || (joined && (int64_t)b->rows * q_heads >= (int64_t)1 << 31))
        return VEDA_ERR_UNSUPPORTED;
    const hipStream_t s = (hipStream_t)stream;
    if (cut.few) return veda::launch_cache_attn_keys(a, bf16, c->head_dim, cut.few, cut.items, s);
    st = veda::launch_cache_attn_rows(a, bf16, c->head_dim, cut.items, s);
    if (st != VEDA_OK || cut.splits == 1) return st;
    const dim3 joins((unsigned)((int64_t)b->rows * q_heads));
    if (bf16 && c->head_dim == 128) hipLaunchKernelGGL((veda::cache_attn_join_splits_kernel<true, 128>), joins, dim3(256), 0, s, a);
    else if (bf16) hipLaunchKernelGGL((veda::cache_attn_join_splits_kernel<true, 64>), joins, dim3(256), 0, s, a);
    else if (c->head_dim == 128) hipLaunchKernelGGL((veda::cache_attn_join_splits_kernel<false, 128>), joins, dim3(256), 0, s, a);
    else hipLaunchKernelGGL((veda::cache_attn_join_splits_kernel<false, 64>), joins, dim3(256), 0, s, a);
    return veda::launch_status("veda_cache_attn_fwd");
}
