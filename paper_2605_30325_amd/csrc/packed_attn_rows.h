// Blocks of many rows over a paged cache held in 4 bits: how a wave's part of a tile comes in, and the whole walk of fp32 rows.  Not part of the public ABI.
#pragma once

#include "cache_attn_keys.h"
#include "packed.h"

namespace veda {

// A tile's segment of kRows rows of either pool, for one wave: C channels of one row of K and of V to a lane (their codes and the byte of their 32).
template <int D, int kRows> struct PackedTile {
    static constexpr int C = kRows * D / 64, W = C / 8;          // channels, and words of codes
    uint32_t k[W], v[W];
    uint32_t ks, vs;
    __device__ static int row(int lane) { return lane * C / D; }
    __device__ static int channel(int lane) { return lane * C % D; }
    // k_at, v_at: the head's place in the page; tok: the segment's first row in it.
    __device__ __forceinline__ void load(const char* k_at, const char* v_at, int tok, int log_page, int lane) {
        const uint32_t code = (uint32_t)(lane * C / 2), scale = (uint32_t)(lane * C / 32);
        const int64_t at = (int64_t)tok * (D / 2), s_at = ((int64_t)(D / 2) << log_page) + (int64_t)tok * (D / 32);
        ks = *reinterpret_cast<const uint8_t*>(k_at + s_at + scale);
        vs = *reinterpret_cast<const uint8_t*>(v_at + s_at + scale);
        packed_words<W>(k_at + at + code, k);
        packed_words<W>(v_at + at + code, v);
    }
    // Whether the lane's key exists; others become zeros, whatever lies there.
    __device__ __forceinline__ void only(bool exists) {
#pragma unroll
        for (int i = 0; i < W; ++i) {
            k[i] = exists ? k[i] : 0u;
            v[i] = exists ? v[i] : 0u;
        }
        ks = exists ? ks : 127u;
        vs = exists ? vs : 127u;
    }
    // Part I of W: a word of K and of V.  k_to, v_to: the segment's first row of either in LDS; kx, vx: the swizzles of the lane's row.
    template <int I> __device__ __forceinline__ void store(char* k_to, char* v_to, int kx, int vx, int lane) const {
        const int at = row(lane) * D * 2, c = packed_chunk<D>(channel(lane) / 8) ^ I;
        *reinterpret_cast<uint4*>(k_to + at + ((c ^ kx) << 4)) = packed_bf16(k[I], packed_power_of(ks));
        *reinterpret_cast<uint4*>(v_to + at + ((c ^ vx) << 4)) = packed_bf16(v[I], packed_power_of(vs));
    }
    template <int I = 0> __device__ __forceinline__ void store_all(char* k_to, char* v_to, int kx, int vx, int lane) const {
        if constexpr (I < W) {
            store<I>(k_to, v_to, kx, vx, lane);
            store_all<I + 1>(k_to, v_to, kx, vx, lane);
        }
    }
};

// fp32 rows.  The cache's values are exact in bf16; Q and the weights come as three bf16 parts each, which hold all 24 bits of an fp32 number, so all
// products are exact and sums are in fp32: three v_mfma_f32_16x16x32_bf16 (48 cycles) stand for eight v_mfma_f32_16x16x4_f32 (256).  A workgroup
// takes 128 rows, 16 to each of its eight waves: with 32 rows three parts of Q, 96 registers, and the sums, 64, leave no room for the rest
// (2464 rows x 12 heads, d = 128, causal behind 2000 keys: 178 us; 420 with 32 rows, and 530 on the fp32 matrix cores).  Reading a tile from LDS
// for 16 rows instead of 32 costs twice the reads, which three products for each have the time for.  What bounds it: the matrix cores and the
// vector instructions of the weights alike, 1.3 us each for a tile of a workgroup, which a wave's chain of products, weights and products
// keeps from overlapping (up to 333 rows of two sequences, 12 heads on 4, up to 2033 keys: 36 us, of which 28 are this walk and 8 the joining).
constexpr int kSplitThreads = 512, kSplitKeys = 64;
constexpr int kSplitWaves = 2;      // to a SIMD, at least: both halves of a tile in flight take 160 registers at d = 128, 120 at 64 (with four, spilled: 45 us, not 36)
template <int D> struct SplitShape {
    static constexpr int kRowB = D * 2, kTile = kSplitKeys * kRowB, kSlot = 2 * kTile + kSplitKeys * 4;      // K, V, and which blocks of V stand for NaN
    __device__ static int k_swizzle(int r) { return D == 128 ? r & 15 : (r >> 1) & 7; }
    __device__ static int v_swizzle(int r) { return packed_v_swizzle<D>(r); }
};
template <int D> constexpr int split_lds() { return 2 * SplitShape<D>::kSlot; }

template <int D>
__device__ __forceinline__ void split_piece(const CacheAttnArgs& a, char* smem, int seq, const SeqRows& sr, int r0, int r_end, int head, const AttnTiles& tiles,
                                            int t_beg, int t_end, int64_t part) {
    typedef SplitShape<D> Sh;
    typedef PackedTile<D, kSplitKeys / 8> Raw;
    constexpr int C = D / 16, kRowB = Sh::kRowB;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), l15 = lane & 15, g = lane >> 4;
    const int n = min(sr.n, a.c.max_new), rows = n * a.group;
    const int w0 = r0 + 16 * wave;
    const bool active = w0 < rows;
    const int r = min(w0 + l15, rows - 1);
    const Seen see = seen_by(a, sr, n, r);
    const int some_lo = __builtin_amdgcn_readlane(see.lo, 0), some_hi = __builtin_amdgcn_readlane(see.hi, 15);
    const int all_lo = __builtin_amdgcn_readlane(see.lo, 15), all_hi = __builtin_amdgcn_readlane(see.hi, 0);
    bf16x8 q[3][D / 32];
    {
        const char* from = a.q + (int64_t)(sr.first + r / a.group) * a.sq_n + (int64_t)(head * a.group + r % a.group) * a.sq_h;
#pragma unroll
        for (int t = 0; t < D / 32; ++t)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const f32x4v x = *reinterpret_cast<const f32x4v*>(from + 128 * t + 32 * g + 16 * h);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    __bf16 p[3];
                    packed_parts(x[e], p);
#pragma unroll
                    for (int u = 0; u < 3; ++u) q[u][t][4 * h + e] = p[u];
                }
            }
    }
    f32x4v o[C];
#pragma unroll
    for (int c = 0; c < C; ++c) o[c] = f32x4v{0.0f, 0.0f, 0.0f, 0.0f};
    float ref = -INFINITY, sub = 0.0f, l = 0.0f;
    uint32_t nan = 0;                      // bit i: the i-th quarter of the channels is NaN

    // Places of the next 64 tiles, one a lane; the wave's segment is 8 keys of each.
    const int64_t head_b = (int64_t)head * (D / 2 + D / 32) << a.c.log_page;
    const int page_mask = (1 << a.c.log_page) - 1, seg = wave * 8;
    const int32_t* table = a.c.table + seq * a.c.table_stride;
    int32_t page = 0;
    uint32_t there = 0;                    // which groups of 16 keys exist
    auto look_up = [&](int t) {
        const int mine = t + lane, tok = tiles.at(mine);
        there = 0;
#pragma unroll
        for (int b = 0; b < kSplitKeys / 16; ++b) {
            const int at = tok + 16 * b, id = mine < t_end && at < sr.len ? table[at >> a.c.log_page] : -1;
            const bool ok = id >= 0 && id < a.c.pages;
            there |= (ok ? 1u : 0u) << b;
            if (b == seg / 16) page = ok ? id : 0;
        }
    };
    Raw raw;
    int raw_t = t_beg, raw_at = 64, raw_key = 0;
    uint32_t raw_exists = 0, next_exists = 0;
    auto load = [&]() __attribute__((always_inline)) {
        if (raw_t >= t_end) return;
        if (raw_at == 64) {
            look_up(raw_t);
            raw_at = 0;
        }
        raw_exists = (uint32_t)__builtin_amdgcn_readlane((int)there, raw_at);
        raw_key = tiles.at(raw_t);
        const int64_t from = __builtin_amdgcn_readlane(page, raw_at) * a.c.page_b + head_b;
        raw.load(a.c.k + from, a.c.v + from, (raw_key + seg) & page_mask, a.c.log_page, lane);
        ++raw_at;
        ++raw_t;
    };
    const int kx = Sh::k_swizzle(seg + Raw::row(lane)), vx = Sh::v_swizzle(seg + Raw::row(lane));
    auto store = [&](int slot) __attribute__((always_inline)) {      // what came in, to a slot
        char* to = smem + slot * Sh::kSlot + seg * kRowB;
        if (raw_exists != (1u << kSplitKeys / 16) - 1u || raw_key + kSplitKeys > sr.len)
            raw.only(((raw_exists >> (seg / 16)) & 1u) && raw_key + seg + Raw::row(lane) < sr.len);
        const bool bad = raw.vs >= kPackedNan;      // zeros in V, and a mark: two lanes hold a quarter of a row
        const uint64_t marks = __ballot(bad);
        if (marks) {
#pragma unroll
            for (int i = 0; i < Raw::W; ++i) raw.v[i] = bad ? 0u : raw.v[i];
            raw.vs = bad ? 127u : raw.vs;
        }
        if (lane < 8) {
            const uint32_t m = (uint32_t)(marks >> (8 * lane));
            *reinterpret_cast<uint32_t*>(smem + slot * Sh::kSlot + 2 * Sh::kTile + (seg + lane) * 4) = (m & 1u) | (m >> 1 & 2u) | (m >> 2 & 4u) | (m >> 3 & 8u);
        }
        raw.store_all(to, to + Sh::kTile, kx, vx, lane);
        next_exists = raw_exists;
    };
    const uint32_t lds = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)smem;
    const uint32_t k_at = (uint32_t)(l15 * kRowB + ((g ^ Sh::k_swizzle(l15)) << 4));
    const int v_key = 4 * g + (l15 >> 2);
    const uint32_t v_at = (uint32_t)(Sh::kTile + v_key * kRowB + ((((l15 & 3) >> 1) ^ Sh::v_swizzle(v_key)) << 4) + 8 * (l15 & 1));

    if (t_beg < t_end) {
        load();
        store(0);
        load();
    }
    int slot = 0;
    for (int t = t_beg; t < t_end; ++t) {
        const uint32_t exists = next_exists;
        const int key0 = tiles.at(t);
        __builtin_amdgcn_s_waitcnt(0xc07f);   // lgkmcnt(0): written, and the other slot has been read
        asm volatile("" ::: "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
        if (t + 1 < t_end) {
            store(slot ^ 1);
            load();
        }
        const uint32_t base = lds + slot * Sh::kSlot;
#pragma unroll 2
        for (int h = 0; h < kSplitKeys / 32; ++h) {
            const int key = key0 + 32 * h;
            const uint32_t ex = (exists >> (2 * h)) & 3u;
            if (!active || key >= some_hi || (key + 32 <= some_lo && key >= a.sinks) || ex == 0) continue;
            const bool full = key + 32 <= all_hi && (key >= all_lo || key + 32 <= a.sinks) && ex == 3u;
            f32x4v s[2];
#pragma unroll
            for (int b = 0; b < 2; ++b) s[b] = f32x4v{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
            for (int i = 0; i < D / 32; ++i) {
                bf16x8 x[2];
#pragma unroll
                for (int b = 0; b < 2; ++b) x[b] = *(lds_bf16x8_p)(uintptr_t)(((base + k_at) ^ (uint32_t)(packed_chunk<D>(4 * i) << 4)) + (32 * h + 16 * b) * kRowB);
#pragma unroll
                for (int u = 2; u >= 0; --u)
#pragma unroll
                    for (int b = 0; b < 2; ++b) s[b] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(x[b], q[u][i], s[b], 0, 0, 0);
            }
            auto sees = [&](int k) __attribute__((always_inline)) { return k < see.hi && (k >= see.lo || k < a.sinks); };
            if (!full) {
#pragma unroll
                for (int b = 0; b < 2; ++b)
#pragma unroll
                    for (int i = 0; i < 4; ++i) s[b][i] = sees(key + 16 * b + 4 * g + i) && ((ex >> b) & 1u) ? s[b][i] : -INFINITY;
            }
            float mx = fmaxf(fmaxf(fmaxf(s[0][0], s[0][1]), fmaxf(s[0][2], s[0][3])), fmaxf(fmaxf(s[1][0], s[1][1]), fmaxf(s[1][2], s[1][3]))) * a.scale_log2;
            if (__any(mx > ref + kAttnSlack)) {
                mx = fmaxf(mx, __shfl_xor(mx, 16));
                mx = fmaxf(mx, __shfl_xor(mx, 32));
                const float up = fmaxf(ref, mx), alpha = up == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(ref - up);
                ref = up;
                sub = up == -INFINITY ? 0.0f : -up;
                l *= alpha;
#pragma unroll
                for (int c = 0; c < C; ++c) o[c] *= alpha;
            }
            bf16x8 p[3];
            float sum = 0.0f;
#pragma unroll
            for (int b = 0; b < 2; ++b)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float w = __builtin_amdgcn_exp2f(__builtin_fmaf(s[b][i], a.scale_log2, sub));
                    sum += w;
                    const float w0 = __uint_as_float(__float_as_uint(w) & 0xffff0000u), rest = w - w0, w1 = __uint_as_float(__float_as_uint(rest) & 0xffff0000u);
                    p[0][4 * b + i] = (__bf16)w0;
                    p[1][4 * b + i] = (__bf16)w1;
                    p[2][4 * b + i] = (__bf16)(rest - w1);
                }
            l += sum;
#pragma unroll
            for (int c = 0; c < C; c += 2) {
                const uint32_t v = base + v_at + 32 * h * kRowB;
                const bf16x8 x[2] = {keys_v_at<D>(v ^ (uint32_t)(packed_chunk<D>(2 * c) << 4)), keys_v_at<D>(v ^ (uint32_t)(packed_chunk<D>(2 * c + 2) << 4))};
#pragma unroll
                for (int j = 0; j < 6; ++j) o[c + j % 2] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(x[j % 2], p[2 - j / 2], o[c + j % 2], 0, 0, 0);
            }
            const uint32_t mark = *reinterpret_cast<const uint32_t*>(smem + slot * Sh::kSlot + 2 * Sh::kTile + (32 * h + (lane & 31)) * 4);
#pragma unroll 1
            for (uint32_t left = (uint32_t)__ballot(mark != 0); left; left &= left - 1) {
                const int k = __ffs((int)left) - 1;
                nan |= sees(key + k) ? (uint32_t)__builtin_amdgcn_readlane((int)mark, k) : 0u;
            }
        }
        slot ^= 1;
    }
    __syncthreads();      // before another piece's values come
    l = keys_sum(l);
    if (w0 + l15 >= r_end) return;
    auto sums = [&](int c) {
        f32x4v x = o[c];
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] = (nan >> (c / (D / 64))) & 1u ? __builtin_nanf("") : x[i];
        return x;
    };
    if (part >= 0) {   // [part][row][D] sums, then [part][row] reference and l
        const int64_t row = part * a.part_rows + 16 * wave + l15;
#pragma unroll
        for (int c = 0; c < C; ++c) *reinterpret_cast<f32x4v*>(a.part + row * D + 16 * c + 4 * g) = sums(c);
        if (g == 0) *reinterpret_cast<float2*>(a.part + rows_pieces(a) * a.part_rows * D + row * 2) = float2{ref, l};
        return;
    }
    const float inv = attn_inverse(a, seq, sr, r, l);
    const int64_t token = sr.first + r / a.group;
    const int qh = head * a.group + r % a.group;
    char* to = a.out + token * a.so_n + (int64_t)qh * a.so_h + 16 * g;
#pragma unroll
    for (int c = 0; c < C; ++c) *reinterpret_cast<f32x4v*>(to + 64 * c) = sums(c) * inv;
    if (a.lse && g == 0) a.lse[(int64_t)qh * a.c.rows + token] = attn_lse(ref, l);
}

}  // namespace veda
