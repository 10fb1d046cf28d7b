// Declarations shared by the kernels of the attention over the paged cache.  Not part of the public ABI.
#pragma once

#include "attn_common.h"
#include "cache.h"

namespace veda {

struct CacheAttnArgs {
    CacheArgs c;
    const char* q;
    char* out;
    float* lse;
    int64_t sq_h, sq_n, so_h, so_n;   // bytes
    int32_t q_heads, group;           // group: query heads of a key head
    int64_t items;                    // blocks of rows of one key head, at most
    int32_t per_seq;                  // see block_of
    int32_t workers;                  // workgroups that share all keys evenly, or 0: one for each block of rows and key head
    int32_t part_rows;                // rows of a block's unfinished sums in the workspace, even
    int32_t block, window, sinks;
    float scale_log2;                 // softmax_scale * log2(e)
    float* part;                      // unfinished sums, and their references and l (see the kernels)
};

typedef __attribute__((ext_vector_type(4))) __bf16 bf16x4;
typedef const __attribute__((address_space(3))) float* lds_f32_ptr;
typedef __attribute__((ext_vector_type(4))) float f32x4v;
typedef const __attribute__((address_space(3))) f32x4v* lds_f32x4_ptr;
typedef const __attribute__((address_space(3))) bf16x8* lds_bf16x8_p;
typedef __attribute__((address_space(3))) bf16x4* lds_bf16x4_p;

constexpr float kAttnSlack = 8.0f;    // log2 units a row maximum may outgrow the reference of its exponentials

// Keys that row r (clamped to the rows there are) of a sequence sees: [lo, hi) and [0, min(sinks, hi)).
struct Seen { int lo, hi; };
__device__ __forceinline__ Seen seen_by(const CacheAttnArgs& a, const SeqRows& sr, int n, int r) {
    const int p = sr.len - sr.n + min(r / a.group, n - 1);
    if (p < 0) return {0, 0};
    const int e = a.block ? (p / a.block + 1) * a.block : sr.len;
    return {a.window ? max(0, e - a.window) : 0, min(e, sr.len)};
}

// A value that is not finite reaches the rows that see its key, and no others, as a count: 1 for +inf, 128 for -inf, 129 for NaN, of at
// most 32 keys, so a sum of them says which there were.  Times 2^14 where the weight has come out as 0: 0 times infinity, NaN, as
// the product itself gives in tiles that all rows see.
constexpr float kCodeNothing = 16384.0f;
__device__ __forceinline__ float attn_code(float x) {
    return (x < INFINITY ? 0.0f : 1.0f) + (x > -INFINITY ? 0.0f : 128.0f);
}
__device__ __forceinline__ float attn_times(float p, bool seen) { return p > 0.0f ? 1.0f : seen ? kCodeNothing : 0.0f; }
__device__ __forceinline__ float attn_decode(float code) {
    const float down = floorf(code * (1.0f / 128.0f));
    const float sum = (code > 128.0f * down ? INFINITY : 0.0f) + (down > 0.0f ? -INFINITY : 0.0f);
    return code >= kCodeNothing ? __builtin_nanf("") : sum;
}

// Whether row r of a sequence sees a key that exists.
__device__ __forceinline__ bool attn_sees(const CacheAttnArgs& a, int seq, const SeqRows& sr, int r) {
    const Seen v = seen_by(a, sr, min(sr.n, a.c.max_new), r);
    const int32_t* table = a.c.table + seq * a.c.table_stride;
    const int sinks = min(a.sinks, v.hi);
    bool found = false;
    for (int tok = sinks > 0 ? 0 : v.lo; tok < v.hi && !found;) {
        const int id = table[tok >> a.c.log_page], next = ((tok >> a.c.log_page) + 1) << a.c.log_page;
        found = id >= 0 && id < a.c.pages;
        tok = next < sinks ? next : max(next, v.lo);
    }
    return found;
}
// 1 / l.  All weights are 0 where a row sees no key, which gives zeros and -inf, and where all its logits are -inf: 0 / 0, NaN.  Their sum
// does not tell these apart, so there, and only there, the table is looked through.
__device__ __forceinline__ float attn_inverse(const CacheAttnArgs& a, int seq, const SeqRows& sr, int r, float l) {
    if (l != 0.0f) return 1.0f / l;
    return attn_sees(a, seq, sr, r) ? __builtin_nanf("") : 0.0f;
}
__device__ __forceinline__ float attn_lse(float ref, float l) { return (ref + __log2f(l)) * kLn2; }

// Tiles of `size` keys that some row of a block sees, as one list: those of the tokens that stay visible, from token 0 on, then those of the
// window, from its first key on, down to a multiple of 16: no 16 keys lie in two pages, and that is all that the loads ask for (tiles
// from multiples of their size on: half a tile more, prompts of up to 4096 tokens with a window of 1024 326 us instead of 320, of 256 149 instead of 144).
struct AttnTiles {
    int size, first, rest, count;   // first: tiles of the one kind; rest: where the others begin
    __device__ __forceinline__ int at(int t) const { return t < first ? t * size : rest + (t - first) * size; }   // its first key
};
__device__ __forceinline__ AttnTiles tiles_seen(const CacheAttnArgs& a, const SeqRows& sr, int n, int r_first, int r_last, int size) {
    const int lo = seen_by(a, sr, n, r_first).lo, hi = seen_by(a, sr, n, r_last).hi;   // both grow from row to row
    AttnTiles t;
    t.size = size;
    t.first = a.window ? (min(a.sinks, hi) + size - 1) / size : 0;
    t.rest = max(t.first * size, lo & ~15);
    t.count = t.first + max(0, (hi - t.rest + size - 1) / size);
    return t;
}

// `total` tiles in equal parts: part p is [begin(p), begin(p + 1)).
struct TileShare {
    int total, parts;
    __device__ __forceinline__ TileShare(int total_, int most, int least) : total(total_), parts(max(1, min(most, (total_ + least - 1) / least))) {}
    __device__ __forceinline__ int begin(int p) const { return (int)((int64_t)p * total / parts); }
    __device__ __forceinline__ int owner(int tile) const { return (int)((((int64_t)tile + 1) * parts + total - 1) / total) - 1; }
};

// Pieces that unfinished sums can come in, at most (see the sharing kernel).
__device__ __forceinline__ int64_t rows_pieces(const CacheAttnArgs& a) { return 2 * (int64_t)a.workers + a.items * a.c.kv_heads; }

// Launches: blocks of 128 rows, or 256 (cache_attn_rows.hip; a.part_rows says so), and blocks of 16 or 32 (cache_attn_keys.hip); and the workgroups of either that
// run at once on the card's 256 compute units.
constexpr int kAttnRows = 128;
constexpr int kRowsShareItems = 256;   // blocks of rows that can be shared out, at most
int attn_rows_places();
int attn_rows_workers(bool bf16);
veda_status launch_cache_attn_rows(const CacheAttnArgs& a, bool bf16, int d, hipStream_t s);
veda_status launch_packed_attn_rows(const CacheAttnArgs& a, bool bf16, int d, hipStream_t s);   // over a cache held in 4 bits
int packed_keys_workers(bool bf16, int d, int size);   // size: rows of a block
veda_status launch_packed_attn_keys(const CacheAttnArgs& a, bool bf16, int d, hipStream_t s);
int attn_keys_workers(bool bf16, int d);
veda_status launch_cache_attn_keys(const CacheAttnArgs& a, bool bf16, int d, hipStream_t s);   // a.part_rows: rows of a block

}  // namespace veda
