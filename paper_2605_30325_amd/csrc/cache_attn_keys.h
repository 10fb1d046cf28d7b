// What the attention kernels for few rows share, over a cache of f32 or bf16 rows and one held in 4 bits: the places of a tile in LDS, how the
// tiles of all sequences are numbered and cut, and the joining of unfinished sums.  Not part of the public ABI.
#pragma once

#include "cache_attn.h"

namespace veda {

typedef __attribute__((ext_vector_type(2))) float f32x2v;

template <bool kBf16, int D> struct KeysTile {
    static constexpr int kRowB = D * (kBf16 ? 2 : 4), kChunks = kRowB / 16;
    static constexpr int kSegRows = kBf16 ? 16 : 8;               // rows of a group of loads: never across a page's end
    static constexpr int kSegLoads = kSegRows * kRowB / 1024;     // 1 KB each
    // Keys of a tile: as many as leave a compute unit's LDS room for three waves with three slots each (fp32, d = 128, with 32 / 16 keys, us:
    // 64 caches of 4096 keys of 8 heads 505 / 445, 33 of up to 2095 of 7 heads 71 / 58, one of 257 of 12 heads, by eight waves, 14.4 / 11.7).
    static constexpr int kKeys = kBf16 || D == 64 ? 32 : 16;
    static constexpr int kGroups = kKeys / 16;
    static constexpr int kSegs = kKeys / kSegRows;
    static constexpr int kSlot = 2 * kKeys * kRowB;               // rows of K, rows of V
    static constexpr int kOutRowB = D * 4 + 16;                   // a row of the sums in LDS
    static constexpr int kLoads = 2 * kSegs * kSegLoads;          // of a tile
    static constexpr int kDepth = 3;                              // slots of a wave that shares: loads run two tiles ahead
    // 16-byte chunk c of row r lies at chunk c ^ swizzle: operand reads of a wave then fall into different banks.
    __device__ static int k_swizzle(int r) { return kBf16 ? (D == 128 ? r & 15 : (r >> 1) & 7) : r & 7; }
    __device__ static int v_swizzle(int r) { return kBf16 ? (D == 128 ? (r & 7) << 1 : ((r >> 1) & 3) << 1) : ((r >> 2) & 3) << 2; }
    // What load j of segment s has on top of the first load's, as address bits.
    __device__ static constexpr uint32_t k_step(int j) { return (uint32_t)j << (kBf16 || D == 64 ? 6 : 5); }
    __device__ static constexpr uint32_t v_step(int s, int j) {
        return kBf16 ? (D == 128 ? (uint32_t)(j & 1) << 7 : 0u) : ((uint32_t)(D == 64 ? j : j >> 1) << 6) ^ ((uint32_t)(s & 1) << 7);
    }
};

// bf16: operand of V for channels 16 c.. of 32 keys, by transposing reads: elements 0-3 are keys 4 g + e, 4-7 keys 16 + 4 g + e.
template <int D> __device__ __forceinline__ bf16x8 keys_v_at(uint32_t at) {
    const bf16x4 x = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds_bf16x4_p)(uintptr_t)at);
    const bf16x4 y = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds_bf16x4_p)(uintptr_t)(at + 16 * (D * 2)));
    return __builtin_shufflevector(x, y, 0, 1, 2, 3, 4, 5, 6, 7);
}
template <int D> __device__ __forceinline__ bf16x8 keys_v(uint32_t v, int c) { return keys_v_at<D>(v ^ (uint32_t)(c << 5)); }
// bf16: a weight goes into its product in two parts, 2^-15 of it off at most (one part: 2^-8, which is as much as the results' own rounding).  The
// matrix cores have the time: us with one / two parts, d = 128: ragged single tokens of 64 streams 193.7 / 193.4, one of a cache of 131,101 105.6 /
// 105.8, 64 of 501 keys 23.9 / 24.2, 512 of 101 51.0 / 51.9; 32 rows of 16 caches of 4100 keys, the dearest, 57.2 / 60.8.
// The first part is the largest value below the weight, so that the rest of a weight above 0 is above 0 too: neither part's product with an
// infinite value is NaN.
__device__ __forceinline__ __bf16 keys_part(float p) {
    return __builtin_bit_cast(__bf16, (uint16_t)(__builtin_elementwise_sub_sat(__builtin_bit_cast(uint32_t, p), 1u) >> 16));
}

// Sum of a row's four lanes.
__device__ __forceinline__ float keys_sum(float x) {
    x += __shfl_xor(x, 16);
    return x + __shfl_xor(x, 32);
}
template <bool kBf16> __device__ __forceinline__ void keys_store(char* dst, f32x4v o) {
    if constexpr (kBf16) {
        bf16x4 x;
#pragma unroll
        for (int e = 0; e < 4; ++e) x[e] = (__bf16)o[e];
        *reinterpret_cast<bf16x4*>(dst) = x;
    } else {
        *reinterpret_cast<f32x4v*>(dst) = o;
    }
}

// Tiles of a sequence in the common row (one that has rows but sees nothing counts as one).
__device__ __forceinline__ int keys_tiles_of(const CacheAttnArgs& a, int s, int size) {
    const SeqRows sr = seq_rows(a.c, s);
    const int n = min(sr.n, a.c.max_new);
    return n == 0 ? 0 : max(1, tiles_seen(a, sr, n, 0, n * a.group - 1, size).count);
}
constexpr int kShareTiles = 8;    // least part of a workgroup: shorter ones are over before their set-up is paid for
// The first 64 sequences' tiles by lane, and the sum over all.
struct KeysCount {
    int size, mine, up_to, total;
    __device__ __forceinline__ KeysCount(const CacheAttnArgs& a, int size_) : size(size_), total(0) {
        for (int s0 = (a.c.seqs - 1) & ~63; s0 >= 0; s0 -= 64) {
            const int s = s0 + (threadIdx.x & 63);
            mine = s < a.c.seqs ? keys_tiles_of(a, s, size) : 0;
            up_to = lanes_up_to(mine);
            total += __builtin_amdgcn_readlane(up_to, 63);
        }
    }
};
// Sequence that tile number `tile` (below the total) falls into, and the number of its first tile.
__device__ __forceinline__ void keys_find(const CacheAttnArgs& a, const KeysCount& count, int tile, int& seq, int& first) {
    int mine = count.mine, up_to = count.up_to;
    first = 0;
    for (int s0 = 0; s0 < a.c.seqs; s0 += 64) {
        if (s0) {
            const int s = s0 + (threadIdx.x & 63);
            mine = s < a.c.seqs ? keys_tiles_of(a, s, count.size) : 0;
            up_to = lanes_up_to(mine);
        }
        const int here = __builtin_amdgcn_readlane(up_to, 63);
        if (tile < first + here) {
            const int at = __popcll(__ballot(first + up_to <= tile));
            seq = s0 + at;
            first += __builtin_amdgcn_readlane(up_to, at) - __builtin_amdgcn_readlane(mine, at);
            return;
        }
        first += here;
    }
    seq = a.c.seqs;
}

struct KeysSeen { int lo, hi, lo_all, hi_all; };   // some row sees keys from lo and below hi, every row those from lo_all and below hi_all

// 64-bit value of another lane, the same for all.
__device__ __forceinline__ int64_t lane_value(int64_t x, int lane) {
    return (int64_t)((uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(uint64_t)x, lane) |
                     (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)((uint64_t)x >> 32), lane) << 32);
}

// Puts the unfinished sums of a (row, query head) together; rows that one workgroup had whole have none.  W waves for each: one
// where there are about as many sequences as parts, more for few long sequences, cut into many; kAhead loads in flight each.
template <bool kBf16, int D, int RB, int W, int kKeys, int kAhead, int kLeast> __global__ __launch_bounds__((W > 8 ? 64 * W : 512)) void cache_attn_join_parts_kernel(CacheAttnArgs a) {
    constexpr int kRows = 16 * RB, V = D / 64;
    __shared__ float sums[W][D + 2];
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, w = wave % W;
    int64_t item;
    if constexpr (W > 8) item = blockIdx.x;
    else item = (int64_t)blockIdx.x * (8 / W) + wave / W;
    const bool is_row = item < (int64_t)a.c.rows * a.q_heads;
    const int token = is_row ? (int)(item / a.q_heads) : -1, qh = (int)(item % a.q_heads);
    // the row's sequence, and its tiles
    int first = 0, each = 0, row = 0, total = 0, seq = 0;
    for (int s0 = 0; s0 < a.c.seqs; s0 += 64) {
        const int s = s0 + lane;
        int mine = 0, i = -1;
        if (s < a.c.seqs) {
            mine = keys_tiles_of(a, s, kKeys);
            const SeqRows sr = seq_rows(a.c, s);
            if (token >= sr.first && token - sr.first < min(sr.n, a.c.max_new)) i = token - sr.first;
        }
        const int up_to = lanes_up_to(mine);
        const uint64_t found = __ballot(i >= 0);
        if (found && each == 0) {
            const int at = __ffsll((long long)found) - 1;
            each = __builtin_amdgcn_readlane(mine, at);
            first = total + __builtin_amdgcn_readlane(up_to, at) - each;
            row = __builtin_amdgcn_readlane(i, at) * a.group + qh % a.group;
            seq = s0 + at;
        }
        total += __builtin_amdgcn_readlane(up_to, 63);
    }
    const TileShare share(total, a.workers / a.c.kv_heads, kLeast);
    const int w0 = each ? share.owner(first) : 0, n = each ? share.owner(first + each - 1) - w0 + 1 : 1;
    if (n == 1) return;   // one workgroup had it all (with W = 8 the same for all waves)
    const float2* ml = reinterpret_cast<const float2*>(a.part + (int64_t)2 * a.workers * kRows * D);
    auto part_row = [&](int j) { return (2 * ((int64_t)(w0 + j) * a.c.kv_heads + qh / a.group) + (j == 0 ? 1 : 0)) * kRows + row; };
    float2 m[kAhead];
    float x[kAhead][V];
    auto get = [&](int j0) {
#pragma unroll
        for (int j = 0; j < kAhead; ++j) {
            const int64_t at = part_row(min(j0 + W * j, n - 1));
            m[j] = ml[at];
#pragma unroll
            for (int c = 0; c < V; ++c) x[j][c] = a.part[at * D + V * lane + c];
        }
    };
    get(w);   // on their way while the common reference is found
    float ref = -INFINITY;
    if constexpr (kAhead > 4) {
        for (int j = lane; j < n; j += 256) {
            float far[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) far[i] = ml[part_row(min(j + 64 * i, n - 1))].x;
#pragma unroll
            for (int i = 0; i < 4; ++i) ref = fmaxf(ref, far[i]);
        }
    } else {
        for (int j = lane; j < n; j += 64) ref = fmaxf(ref, ml[part_row(j)].x);
    }
#pragma unroll
    for (int x = 32; x >= 1; x >>= 1) ref = fmaxf(ref, __shfl_xor(ref, x));
    float l = 0.0f, o[V];
#pragma unroll
    for (int c = 0; c < V; ++c) o[c] = 0.0f;
    for (int j0 = w; j0 < n; j0 += kAhead * W) {
        if (j0 != w) get(j0);
#pragma unroll
        for (int j = 0; j < kAhead; ++j) {
            if (j0 + W * j >= n) continue;
            const float f = m[j].x == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(m[j].x - ref);   // -inf: the sums are 0 or NaN
            l += f * m[j].y;
#pragma unroll
            for (int c = 0; c < V; ++c) o[c] += f * x[j][c];
        }
    }
    if constexpr (W > 1) {
#pragma unroll
        for (int c = 0; c < V; ++c) sums[w][V * lane + c] = o[c];
        if (lane == 0) sums[w][D] = l;
        __syncthreads();
        if (w != 0) return;
        l = 0.0f;
#pragma unroll
        for (int c = 0; c < V; ++c) o[c] = 0.0f;
#pragma unroll
        for (int x = 0; x < W; ++x) {
            l += sums[x][D];
#pragma unroll
            for (int c = 0; c < V; ++c) o[c] += sums[x][V * lane + c];
        }
    }
    const float inv = l != 0.0f ? 1.0f / l : attn_inverse(a, seq, seq_rows(a.c, seq), row, l);
    char* dst = a.out + token * a.so_n + (int64_t)qh * a.so_h;
#pragma unroll
    for (int c = 0; c < V; ++c) {
        if constexpr (kBf16) reinterpret_cast<__bf16*>(dst)[V * lane + c] = (__bf16)(o[c] * inv);
        else reinterpret_cast<float*>(dst)[V * lane + c] = o[c] * inv;
    }
    if (a.lse && lane == 0) a.lse[(int64_t)qh * a.c.rows + token] = attn_lse(ref, l);
}

}  // namespace veda
