// Attention over a paged cache held in 4 bits, few rows for each key head (single tokens and small chunks).
//
// The mathematics, the numbering of tiles, the shares and the joining are those of cache_attn_keys.hip; what a wave does with a tile of 32 keys
// is not.  Codes come straight into registers: four lanes hold a row, each the codes of a quarter of its channels, and as the order of channels in
// a sum of products is free, a lane's codes of K, turned into bf16 eight at a time, are operands as they stand (Q is read in the same order).
// V has to change sides (its products run over keys), so its values go through the wave's own 32 rows of LDS, by transposing reads.  All values
// are exact in bf16; fp32 rows come as three bf16 parts of Q and of the weights (together their 24 bits), with fp32 accumulation.
//
// A byte read is worth four times as many products as in a bf16 cache, so here latency and instructions stand closer to memory than there: no
// barrier, no tile of raw codes in LDS, and as many waves to a compute unit as registers allow.
//
// What bounds it: 64 single tokens of 32 heads on 8, up to 8192 ragged keys, d = 128, bf16, read 285 MB in 61 us of walk (4.7 TB/s; 5 us before the first tile; the
// instructions alone take 51) and 6 of joining; one of 40 heads on 131,101 keys 142 MB in 33 and 11.  fp32, where six products stand for two and a weight is cut in
// three: 64 up to 4000 ragged keys read 130 MB in 42 us of walk (3.1 TB/s; bf16 35) and 5 of joining, vector instructions 34 % and matrix pipes 21 % busy, waves waiting
// for memory 28 % and for their turn 25 % of their time: two to a SIMD do not overlap these.
#include "cache_attn_keys.h"
#include "packed.h"

namespace veda {

template <int D, int G> struct PackedKeys {
    // Keys of a tile in groups of 16, and the least tiles of a share.
    static constexpr int kKeys = 16 * G, kLeast = 16 / G;
    static constexpr int W = D / 32;                     // words of codes a lane has of 16 keys
    static constexpr int kRowB = D / 2, kScaleB = D / 32;
    static constexpr int kSlot = kKeys * D * 2;          // V in LDS
    static constexpr int kOutRowB = D * 4 + 16;          // a row of the sums in LDS
};

template <bool kBf16, int D, int RB> struct PackedRow {
    static constexpr int kQ = kBf16 ? 1 : 3;             // bf16 parts of Q
    f32x4v o[RB][D / 16];
    bf16x8 q[kQ][RB][D / 32];
    float ref[RB], sub[RB], l[RB];   // reference of the exponentials (log2 units), 0 or -ref, this lane's sum
    float scale[RB];                 // of the logits
    int lo[RB], hi[RB];              // visible keys
    uint32_t nan[RB];                // bit i: the i-th quarter of the channels is NaN
    __device__ __forceinline__ f32x4v sums(int rb, int c) const {      // of channels 16 c + 4 g + 0..3
        f32x4v x = o[rb][c];
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] = (nan[rb] >> (c / (D / 64))) & 1u ? __builtin_nanf("") : x[i];
        return x;
    }
};

// Waves to a SIMD that the registers are to leave room for.
template <bool kBf16, int D, int RB> constexpr int packed_waves() { return RB == 2 ? (kBf16 || D == 64 ? 2 : 1) : D == 64 ? 3 : 2; }

// The sharing kernel: tiles of a wave in flight, and groups of 16 keys of each.  Two of 32 keys are as many bytes as one of 64, asked for a whole tile earlier; with
// bf16 and d = 64 instructions bound the walk, and a larger tile has fewer, and for 32 rows there are no registers (us with two of 32 / one of 64, ragged single
// tokens of 64 streams of 32 heads on 8, d = 128, 65.5 / 67.5, one of 40 heads on 131,101 keys 40.9 / 42.0; fp32, 64 streams up to 4000 keys 46.3 / 48.4, d = 64 34.4 / 37.2;
// bf16, d = 64, up to 8192 keys 43.8 / 42.4).  From memory, not the 256 MB beside it, the first two take 71 and 44 either way.
template <bool kBf16, int D, int RB> constexpr int packed_ring() { return RB == 2 || (kBf16 && D == 64) ? 1 : 2; }
template <bool kBf16, int D, int RB> constexpr int packed_groups() { return RB == 2 || packed_ring<kBf16, D, RB>() == 2 ? 2 : 4; }

// A lane's part of a tile: of its K row (l15), and of V, where lane / 4 is the key.
template <int D, int G> struct PackedRaw {
    uint32_t k[G][D / 32], v[G][D / 32];
    uint32_t ks[G], vs[G];                               // four bytes s, the lane's among them
};
template <int D, int G> struct PackedLane {
    typedef PackedKeys<D, G> P;
    uint32_t k_code, k_scale, v_code, v_scale;           // what the lane adds to addresses in a pool
    uint32_t v_to, v_at;                                 // its places in LDS: where its part of V goes, and its operand's
    uint32_t k_shift, v_shift;                           // of the lane's byte in its four
    int lane, l15, g;
    __device__ __forceinline__ explicit PackedLane(int lane_) : lane(lane_), l15(lane_ & 15), g(lane_ >> 4) {
        k_code = (uint32_t)(l15 * P::kRowB + g * (D / 8));
        k_scale = (uint32_t)(l15 * P::kScaleB + g * (D / 4) / 32);
        k_shift = 8 * (k_scale & 3);
        k_scale &= ~3u;
        v_code = (uint32_t)(lane * (D / 8));
        v_scale = (uint32_t)((lane >> 2) * P::kScaleB + (lane & 3) * (D / 4) / 32);
        v_shift = 8 * (v_scale & 3);
        v_scale &= ~3u;
        v_to = (uint32_t)((lane >> 2) * D * 2 + ((packed_chunk<D>((lane & 3) * (D / 32)) ^ packed_v_swizzle<D>(lane >> 2)) << 4));
        const int key = 4 * g + (l15 >> 2);
        v_at = (uint32_t)(key * D * 2 + ((((l15 & 3) >> 1) ^ packed_v_swizzle<D>(key)) << 4) + 8 * (l15 & 1));
    }
    // The same place for all lanes, in scalar registers, and what a lane adds to it.  (An address in global memory, or the loads would be flat ones, which are
    // waited for all together.)
    typedef const __attribute__((address_space(1))) char* Global;
    __device__ static __forceinline__ Global at(const char* all, uint32_t lane_part) {
        uint64_t x = (uint64_t)(uintptr_t)all;
        asm("" : "+s"(x));
        return (Global)(uintptr_t)x + lane_part;
    }
    template <int W> __device__ static __forceinline__ void words(Global p, uint32_t (&w)[W]) {
        typedef __attribute__((ext_vector_type(W == 1 ? 2 : W))) uint32_t Words;
        if constexpr (W == 1) {
            w[0] = *(const __attribute__((address_space(1))) uint32_t*)p;
        } else {
            const Words x = *(const __attribute__((address_space(1))) Words*)p;
#pragma unroll
            for (int i = 0; i < W; ++i) w[i] = x[i];
        }
    }
    // base: the head's place in the pools, tok: the first of 16 keys in the page.
    __device__ __forceinline__ void load(const CacheArgs& c, PackedRaw<D, G>& r, int b, int64_t base, int tok) const {
        const int64_t code = base + tok * P::kRowB, scale = base + ((int64_t)P::kRowB << c.log_page) + tok * P::kScaleB;
        words(at(c.k + code, k_code), r.k[b]);
        words(at(c.v + code, v_code), r.v[b]);
        r.ks[b] = *(const __attribute__((address_space(1))) uint32_t*)at(c.k + scale, k_scale);
        r.vs[b] = *(const __attribute__((address_space(1))) uint32_t*)at(c.v + scale, v_scale);
    }
};

// Where 16 keys from token `tok` on begin: their head's place in the pools and their number in the page; false if they do not exist.
template <int D> __device__ __forceinline__ bool packed_from(const CacheArgs& c, const int32_t* table, int len, int64_t head_b, int tok, int64_t& base, int& at) {
    const int id = tok < len ? table[tok >> c.log_page] : -1;
    const bool ok = id >= 0 && id < c.pages;
    base = ok ? id * c.page_b + head_b : head_b;   // any place in the pool will do
    at = ok ? tok & ((1 << c.log_page) - 1) : 0;
    return ok;
}

// The rows of a block: what they see and ask for, and no sums yet.
template <bool kBf16, int D, int RB>
__device__ __forceinline__ KeysSeen packed_rows_of(const CacheAttnArgs& a, PackedRow<kBf16, D, RB>& st, const SeqRows& sr, int n, int head, int r0, int r_end,
                                                   int l15, int g) {
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) {
        const int r = min(r0 + 16 * rb + l15, r_end - 1);
        const Seen see = seen_by(a, sr, n, r);
        st.lo[rb] = see.lo;
        st.hi[rb] = see.hi;
        const char* q = a.q + (int64_t)(sr.first + r / a.group) * a.sq_n + (int64_t)(head * a.group + r % a.group) * a.sq_h;
        st.scale[rb] = a.scale_log2;
        if constexpr (kBf16) {
#pragma unroll
            for (int t = 0; t < D / 32; ++t) st.q[0][rb][t] = *reinterpret_cast<const bf16x8*>(q + g * (D / 2) + 16 * t);
        } else {
#pragma unroll
            for (int t = 0; t < D / 32; ++t)
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const f32x4v x = *reinterpret_cast<const f32x4v*>(q + g * D + 32 * t + 16 * h);
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        __bf16 p[3];
                        packed_parts(x[e], p);
#pragma unroll
                        for (int u = 0; u < 3; ++u) st.q[u][rb][t][4 * h + e] = p[u];
                    }
                }
        }
#pragma unroll
        for (int c = 0; c < D / 16; ++c) st.o[rb][c] = f32x4v{0.0f, 0.0f, 0.0f, 0.0f};
        st.ref[rb] = -INFINITY;
        st.sub[rb] = st.l[rb] = 0.0f;
        st.nan[rb] = 0;
    }
    // Q is waited for here: left to its first use, in the loop over tiles, the wait would be there, and every tile would wait for the next one's loads.
#pragma unroll
    for (int u = 0; u < PackedRow<kBf16, D, RB>::kQ; ++u)
#pragma unroll
        for (int rb = 0; rb < RB; ++rb)
#pragma unroll
            for (int t = 0; t < D / 32; ++t) asm volatile("" : "+v"(st.q[u][rb][t]));
    return {__builtin_amdgcn_readlane(st.lo[0], 0), __builtin_amdgcn_readlane(st.hi[RB - 1], 15), __builtin_amdgcn_readlane(st.lo[RB - 1], 15),
            __builtin_amdgcn_readlane(st.hi[0], 0)};
}

// A tile of keys from key0 on for one wave, in two halves between which the next tile's codes are asked for, into the registers that the first
// half is done with.  exists: bit b = keys 16 b .. 16 b + 15 exist; len: the sequence's tokens.
template <int G> struct PackedStep {
    int key0;
    uint32_t exists;
    bool some, full, odd;    // some row sees some keys; every row sees all; blocks of V stand for NaN
    uint64_t nans[G];        // the lanes that have some
};
// V goes to its places in LDS (at smem), scores are formed.
template <bool kBf16, int D, int RB, int G>
__device__ __forceinline__ void packed_scores(const CacheAttnArgs& a, const PackedRow<kBf16, D, RB>& st, const KeysSeen& see, const PackedLane<D, G>& ln, PackedRaw<D, G>& raw,
                                              char* smem, int len, PackedStep<G>& step, f32x4v (&s)[RB][G]) {
    constexpr int W = D / 32, kQ = PackedRow<kBf16, D, RB>::kQ;
    const int key0 = step.key0, end = key0 + 16 * G;
    const uint32_t exists = step.exists;
    step.some = !(key0 >= see.hi || (end <= see.lo && key0 >= a.sinks) || exists == 0);
    if (!step.some) return;
    step.full = end <= see.hi_all && (key0 >= see.lo_all || end <= a.sinks) && exists == (1u << G) - 1u;

    // V to its places; zeros for keys that do not exist, whatever lies there, and for blocks that stand for NaN (odd, nans: the lanes that have some)
    uint32_t most = 0, ks[G], vs[G];
#pragma unroll
    for (int b = 0; b < G; ++b) {
        ks[b] = raw.ks[b] >> ln.k_shift & 255u;
        vs[b] = raw.vs[b] >> ln.v_shift & 255u;
        most = max(most, vs[b]);
        step.nans[b] = 0;
    }
    step.odd = __any(most >= kPackedNan);
    if (exists != (1u << G) - 1u || end > len || step.odd) {
#pragma unroll
        for (int b = 0; b < G; ++b) {
            const bool there = ((exists >> b) & 1u) && key0 + 16 * b + (ln.lane >> 2) < len, nan = there && vs[b] >= kPackedNan;
            step.nans[b] = __ballot(nan);
#pragma unroll
            for (int i = 0; i < W; ++i) raw.v[b][i] = there && !nan ? raw.v[b][i] : 0u;
            vs[b] = there && !nan ? vs[b] : 127u;
        }
    }
#pragma unroll
    for (int b = 0; b < G; ++b)
#pragma unroll
        for (int i = 0; i < W; ++i)
            *reinterpret_cast<uint4*>(smem + ((ln.v_to ^ (uint32_t)(i << 4)) + b * 16 * D * 2)) = packed_bf16(raw.v[b][i], packed_power(vs[b]));
    asm volatile("" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);

#pragma unroll
    for (int rb = 0; rb < RB; ++rb)
#pragma unroll
        for (int b = 0; b < G; ++b) s[rb][b] = f32x4v{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int t = 0; t < W; ++t)
#pragma unroll
        for (int b = 0; b < G; ++b) {
            const bf16x8 x = __builtin_bit_cast(bf16x8, packed_bf16(raw.k[b][t], packed_power_of(ks[b])));
#pragma unroll
            for (int u = kQ - 1; u >= 0; --u)
#pragma unroll
                for (int rb = 0; rb < RB; ++rb) s[rb][b] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(x, st.q[u][rb][t], s[rb][b], 0, 0, 0);
        }
}
// Weights, and their products with V (at v in LDS).
template <bool kBf16, int D, int RB, int G>
__device__ __forceinline__ void packed_values(const CacheAttnArgs& a, PackedRow<kBf16, D, RB>& st, const PackedLane<D, G>& ln, uint32_t v, const PackedStep<G>& step,
                                              f32x4v (&s)[RB][G]) {
    constexpr int C = D / 16, kP = kBf16 ? 2 : 3;
    const int key0 = step.key0;
    const uint32_t exists = step.exists;
    if (!step.some) return;
    auto seen = [&](int rb, int b, int i) __attribute__((always_inline)) {
        const int key = key0 + 16 * b + 4 * ln.g + i;
        return key < st.hi[rb] && (key >= st.lo[rb] || key < a.sinks) && ((exists >> b) & 1u);
    };
    float mx[RB];
    bool grown = false;
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) {
        if (!step.full) {
#pragma unroll
            for (int b = 0; b < G; ++b)
#pragma unroll
                for (int i = 0; i < 4; ++i) s[rb][b][i] = seen(rb, b, i) ? s[rb][b][i] : -INFINITY;
        }
        float m = s[rb][0][0];
#pragma unroll
        for (int b = 0; b < G; ++b)
#pragma unroll
            for (int i = 0; i < 4; ++i) m = fmaxf(m, s[rb][b][i]);
        mx[rb] = m * st.scale[rb];
        grown = grown || mx[rb] > st.ref[rb] + kAttnSlack;
    }
    if (__any(grown)) {
#pragma unroll
        for (int rb = 0; rb < RB; ++rb) {
            float m = fmaxf(mx[rb], __shfl_xor(mx[rb], 16));
            m = fmaxf(m, __shfl_xor(m, 32));
            const float ref = fmaxf(st.ref[rb], m);
            const float alpha = ref == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(st.ref[rb] - ref);
            st.ref[rb] = ref;
            st.sub[rb] = ref == -INFINITY ? 0.0f : -ref;
            st.l[rb] *= alpha;
#pragma unroll
            for (int c = 0; c < C; ++c) st.o[rb][c] *= alpha;
        }
    }
    bf16x8 p[G / 2][kP][RB];
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) {
        float sum = 0.0f;
#pragma unroll
        for (int b = 0; b < G; ++b)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int h = b / 2, e = 4 * (b % 2) + i;
                const float w = __builtin_amdgcn_exp2f(__builtin_fmaf(s[rb][b][i], st.scale[rb], st.sub[rb]));
                sum += w;
                // the first part below the weight, so that what is left of a weight above 0 is above 0 too (keys_part)
                p[h][0][rb][e] = keys_part(w);
                const float rest = w - (float)p[h][0][rb][e];
                if constexpr (kP == 2) {
                    p[h][1][rb][e] = (__bf16)rest;
                } else {
                    const float second = __uint_as_float(__float_as_uint(rest) & 0xffff0000u);
                    p[h][1][rb][e] = (__bf16)second;
                    p[h][kP - 1][rb][e] = (__bf16)(rest - second);
                }
            }
        st.l[rb] += sum;
    }
#pragma unroll
    for (int h = 0; h < G / 2; ++h)
#pragma unroll
        for (int c = 0; c < C; c += 2) {   // two at a time, so that a sum's next product is not the one right behind it
            const uint32_t at = v + h * 32 * D * 2;
            const bf16x8 x[2] = {keys_v_at<D>(at ^ (uint32_t)(packed_chunk<D>(2 * c) << 4)), keys_v_at<D>(at ^ (uint32_t)(packed_chunk<D>(2 * c + 2) << 4))};
#pragma unroll
            for (int j = 0; j < 2 * kP * RB; ++j) {
                const int i = c + j % 2, rb = j / 2 % RB, u = kP - 1 - j / 2 / RB;
                st.o[rb][i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(x[j % 2], p[h][u][rb], st.o[rb][i], 0, 0, 0);
            }
            if (c % 4 == 2) __builtin_amdgcn_sched_barrier(0);   // or every operand is read at once, into registers that are not there
        }
    if (step.odd) {   // NaN for the rows that see such a block's key, and for no others
#pragma unroll
        for (int b = 0; b < G; ++b)
#pragma unroll 1
            for (uint64_t left = step.nans[b]; left; left &= left - 1) {
                const int from = __ffsll((long long)left) - 1, key = key0 + 16 * b + (from >> 2);
#pragma unroll
                for (int rb = 0; rb < RB; ++rb) st.nan[rb] |= key < st.hi[rb] && (key >= st.lo[rb] || key < a.sinks) ? 1u << (from & 3) : 0u;
            }
    }
    asm volatile("" ::: "memory");
}

// Places of 64 tiles, one tile a lane: looked up together, so that no step waits for the table.
template <int D, int G> struct PackedPlaces {
    int64_t base[G];
    int info;      // which of the groups of 16 keys exist (bits 0..), and their numbers in their pages (16 at a time: four bits from 8 on)
    __device__ __forceinline__ void find(const CacheArgs& c, const int32_t* table, int len, int64_t head_b, int tok) {
        info = 0;
#pragma unroll
        for (int b = 0; b < G; ++b) {
            int at;
            const bool ok = packed_from<D>(c, table, len, head_b, tok + 16 * b, base[b], at);
            info |= (ok ? 1 << b : 0) | (at >> 4) << (8 + 4 * b);
        }
    }
    // asks for the tile of lane `at`; returns which keys exist
    __device__ __forceinline__ uint32_t ask(const CacheArgs& c, const PackedLane<D, G>& ln, PackedRaw<D, G>& raw, int at) const {
        const int x = __builtin_amdgcn_readlane(info, at);
#pragma unroll
        for (int b = 0; b < G; ++b) ln.load(c, raw, b, lane_value(base[b], at), (x >> (8 + 4 * b) & 15) << 4);
        return (uint32_t)x & ((1u << G) - 1u);
    }
};

// Short caches: a workgroup for each (block of rows, key head), whose waves take its tiles in turn: eight of them, four where workgroups are more than compute
// units, two where they are more than three times as many.  32 fp32 rows of 128 channels want more registers than two waves to a SIMD leave (packed_waves), and spill 82 or 83
// (8 tokens of 4 query heads a key head, us: one cache of 2 heads, 500 keys 22, 2000 48; 64 of 8, 500 48, 1000 72; bf16 rows, which spill none, 12, 24, 19 and 27).
template <bool kBf16, int D, int RB, int G, int kWaves> __global__ __launch_bounds__(64 * kWaves, 2) void packed_attn_keys_kernel(CacheAttnArgs a) {
    typedef PackedKeys<D, G> P;
    constexpr int kRows = 16 * RB, kEs = kBf16 ? 2 : 4;
    extern __shared__ __align__(1024) char smem[];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const PackedLane<D, G> ln(lane);
    char* mine = smem + wave * P::kSlot;
    const uint32_t v = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)smem + wave * P::kSlot + ln.v_at;
    RowBlock block;
    if (!block_of(a.c, a.group, kRows, a.per_seq, blockIdx.x / a.c.kv_heads, block)) return;
    const int head = blockIdx.x % a.c.kv_heads, r0 = block.block * kRows;
    const SeqRows sr = block.rows;
    const int n = min(sr.n, a.c.max_new), r_end = min(n * a.group, r0 + kRows);
    const AttnTiles tiles = tiles_seen(a, sr, n, r0, r_end - 1, P::kKeys);
    const int32_t* table = a.c.table + block.seq * a.c.table_stride;
    const int64_t head_b = (int64_t)head * (P::kRowB + P::kScaleB) << a.c.log_page;

    PackedPlaces<D, G> places;
    PackedRaw<D, G> raw;
    uint32_t exists = 0;
    if (wave < tiles.count) {
        places.find(a.c, table, sr.len, head_b, tiles.at(min(wave + lane * kWaves, tiles.count - 1)));
        exists = places.ask(a.c, ln, raw, 0);
    }
    PackedRow<kBf16, D, RB> st;
    const KeysSeen see = packed_rows_of<kBf16, D, RB>(a, st, sr, n, head, r0, r_end, ln.l15, ln.g);
    int at = 0;
    for (int t = wave; t < tiles.count; t += kWaves) {
        PackedStep<G> step{tiles.at(t), exists};
        f32x4v sc[RB][G];
        packed_scores<kBf16, D, RB, G>(a, st, see, ln, raw, mine, sr.len, step, sc);
        if (t + kWaves < tiles.count) {
            if (++at == 64) {
                places.find(a.c, table, sr.len, head_b, tiles.at(min(t + kWaves + lane * kWaves, tiles.count - 1)));
                at = 0;
            }
            exists = places.ask(a.c, ln, raw, at);
        }
        packed_values<kBf16, D, RB, G>(a, st, ln, v, step, sc);
    }

    // Sums of the waves, put together row by row.  A lane holds channels 16 c + 4 g + 0..3 of its row.
    __syncthreads();
    float* ml = reinterpret_cast<float*>(smem + kWaves * kRows * P::kOutRowB);   // [wave][row][2]
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) {
        const int row = wave * kRows + 16 * rb + ln.l15;
        const float l = keys_sum(st.l[rb]);
#pragma unroll
        for (int c = 0; c < D / 16; ++c) *reinterpret_cast<f32x4v*>(smem + row * P::kOutRowB + (16 * c + 4 * ln.g) * 4) = st.sums(rb, c);
        if (ln.g == 0) {
            ml[2 * row] = st.ref[rb];
            ml[2 * row + 1] = l;
        }
    }
    __syncthreads();
    for (int i = tid; i < (r_end - r0) * (D / 4); i += 64 * kWaves) {
        const int rr = i / (D / 4), ch = 4 * (i % (D / 4)), row = r0 + rr;
        float ref = -INFINITY, l = 0.0f;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) ref = fmaxf(ref, ml[2 * (w * kRows + rr)]);
        f32x4v o = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int w = 0; w < kWaves; ++w) {
            const float m = ml[2 * (w * kRows + rr)], lw = ml[2 * (w * kRows + rr) + 1];
            const float f = m == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(m - ref);   // -inf: the sums are 0 or NaN
            l += f * lw;
            o += f * *reinterpret_cast<const f32x4v*>(smem + (w * kRows + rr) * P::kOutRowB + ch * 4);
        }
        const int64_t token = sr.first + row / a.group;
        const int qh = head * a.group + row % a.group;
        keys_store<kBf16>(a.out + token * a.so_n + (int64_t)qh * a.so_h + ch * kEs, o * attn_inverse(a, block.seq, sr, row, l));
        if (a.lse && ch == 0) a.lse[(int64_t)qh * a.c.rows + token] = attn_lse(ref, l);
    }
}

// Long caches: every wave is a workgroup and takes one key head of an equal part [now, end) of the common row of tiles, sequence by sequence.
template <bool kBf16, int D, int RB, int G> __global__ __launch_bounds__(64, (packed_waves<kBf16, D, RB>())) void packed_attn_share_kernel(CacheAttnArgs a) {
    typedef PackedKeys<D, G> P;
    constexpr int kRows = 16 * RB, kEs = kBf16 ? 2 : 4;
    extern __shared__ __align__(1024) char smem[];
    const int lane = threadIdx.x;
    const PackedLane<D, G> ln(lane);
    const uint32_t v = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)smem + ln.v_at;
    const KeysCount count(a, P::kKeys);
    const TileShare share(count.total, a.workers / a.c.kv_heads, P::kLeast);
    const int head = blockIdx.x % a.c.kv_heads, mine = blockIdx.x / a.c.kv_heads;
    if (mine >= share.parts || share.total == 0) return;
    int now = share.begin(mine);
    const int end = share.begin(mine + 1);
    if (now >= end) return;
    const int64_t head_b = (int64_t)head * (P::kRowB + P::kScaleB) << a.c.log_page;

    struct Place {          // a sequence, and the numbers of its tiles
        int seq, first, each;
        SeqRows sr;
        AttnTiles tiles;
    };
    auto enter = [&](Place& p, int seq, int first) {   // the first sequence from seq on that has rows
        p.first = first;
        p.each = 0;
        for (p.seq = seq; p.seq < a.c.seqs; ++p.seq) {
            p.sr = seq_rows(a.c, p.seq);
            const int n = min(p.sr.n, a.c.max_new);
            if (n == 0) continue;
            p.tiles = tiles_seen(a, p.sr, n, 0, n * a.group - 1, P::kKeys);
            p.each = max(1, p.tiles.count);
            return;
        }
    };
    Place here, ahead;
    {
        int seq, first;
        keys_find(a, count, now, seq, first);
        enter(here, seq, first);
    }
    ahead = here;
    // Places of the next 64 tiles, whichever sequences they belong to.
    PackedPlaces<D, G> places;
    auto look_up = [&](int x) {
        const int at = x + lane;
#pragma unroll
        for (int b = 0; b < G; ++b) places.base[b] = head_b;
        places.info = 0;
        while (ahead.each) {
            const int last = ahead.first + ahead.each, t = at - ahead.first;
            if (t >= 0 && at < last && at < end)
                places.find(a.c, a.c.table + ahead.seq * a.c.table_stride, t < ahead.tiles.count ? ahead.sr.len : 0, head_b, ahead.tiles.at(t));
            if (last >= min(x + 64, end)) break;
            enter(ahead, ahead.seq + 1, last);
        }
    };
    constexpr int kRing = packed_ring<kBf16, D, RB>();
    int asked = now, at = 64;
    PackedRaw<D, G> raw[kRing];
    uint32_t exists[kRing] = {};
    // Behind the last tile too, some place again: were loads left out on any path, the wait for one tile could not leave the next one's in flight.
    auto ask = [&](int i) __attribute__((always_inline)) {
        if (at == 64 && asked < end) {
            look_up(asked);
            at = 0;
        }
        exists[i] = places.ask(a.c, ln, raw[i], min(at, 63));
        ++at;
        ++asked;
    };
#pragma unroll
    for (int i = 0; i < kRing; ++i) ask(i);
    while (now < end && here.each) {
        const SeqRows sr = here.sr;
        const int n = min(sr.n, a.c.max_new), rows = n * a.group;
        const int t_beg = now - here.first, stop = min(end, here.first + here.each);
        PackedRow<kBf16, D, RB> st;
        const KeysSeen see = packed_rows_of<kBf16, D, RB>(a, st, sr, n, head, 0, rows, ln.l15, ln.g);
        auto go = [&](int i) __attribute__((always_inline)) {      // the next tile, which is in raw[i]
            PackedStep<G> step{here.tiles.at(now - here.first), exists[i]};
            f32x4v sc[RB][G];
            packed_scores<kBf16, D, RB, G>(a, st, see, ln, raw[i], smem, sr.len, step, sc);
            ask(i);
            packed_values<kBf16, D, RB, G>(a, st, ln, v, step, sc);
            ++now;
        };
        // (A loop that can be left in its middle would wait for all loads at its top: the compiler lets every way out end in one place with the way back.)
        for (int rounds = (stop - now) / kRing; rounds > 0; --rounds) {
#pragma unroll
            for (int i = 0; i < kRing; ++i) go(i);
        }
        if constexpr (kRing == 2) {
            if (now < stop) {
                go(0);
                const PackedRaw<D, G> x = raw[0];     // the next tile is in the other one
                raw[0] = raw[1];
                raw[1] = x;
                const uint32_t e = exists[0];
                exists[0] = exists[1];
                exists[1] = e;
            }
        }
        // The sums: finished, or to the workspace, [part][row][D] and then [part][row] reference and l.
        const bool whole = t_beg == 0 && stop == here.first + here.each;
        const int64_t part = 2 * (int64_t)blockIdx.x + (t_beg == 0 ? 1 : 0);   // begun by another workgroup, or here
#pragma unroll
        for (int rb = 0; rb < RB; ++rb) {
            const int row = 16 * rb + ln.l15;
            const float l = keys_sum(st.l[rb]);
            if (row >= rows) continue;
            if (!whole) {
                float* po = a.part + (part * kRows + row) * D + 4 * ln.g;
#pragma unroll
                for (int c = 0; c < D / 16; ++c) *reinterpret_cast<f32x4v*>(po + 16 * c) = st.sums(rb, c);
                if (ln.g == 0) *reinterpret_cast<f32x2v*>(a.part + (int64_t)2 * a.workers * kRows * D + (part * kRows + row) * 2) = f32x2v{st.ref[rb], l};
                continue;
            }
            const int64_t token = sr.first + row / a.group;
            const int qh = head * a.group + row % a.group;
            char* dst = a.out + token * a.so_n + (int64_t)qh * a.so_h + 4 * ln.g * kEs;
            const float inv = attn_inverse(a, here.seq, sr, row, l);
#pragma unroll
            for (int c = 0; c < D / 16; ++c) keys_store<kBf16>(dst + 16 * c * kEs, st.sums(rb, c) * inv);
            if (a.lse && ln.g == 0) a.lse[(int64_t)qh * a.c.rows + token] = attn_lse(st.ref[rb], l);
        }
        if (now == here.first + here.each) enter(here, here.seq + 1, now);
    }
}

// Waves to a compute unit: what registers and LDS leave room for.
template <bool kBf16, int D> static int packed_fit(int size) { return 256 * 4 * (size == 16 ? packed_waves<kBf16, D, 1>() : packed_waves<kBf16, D, 2>()); }
int packed_keys_workers(bool bf16, int d, int size) {
    if (bf16) return d == 128 ? packed_fit<true, 128>(size) : packed_fit<true, 64>(size);
    return d == 128 ? packed_fit<false, 128>(size) : packed_fit<false, 64>(size);
}

template <bool kBf16, int D, int RB, int G, int kWaves> static veda_status launch_short(const CacheAttnArgs& a, hipStream_t s) {
    typedef PackedKeys<D, G> P;
    constexpr int kSums = kWaves * 16 * RB * (P::kOutRowB + 8), kTiles = kWaves * P::kSlot, kLds = kTiles > kSums ? kTiles : kSums;
    static_assert(kLds <= 160 * 1024, "what a compute unit has");
    auto kern = packed_attn_keys_kernel<kBf16, D, RB, G, kWaves>;
    if (kLds > 64 * 1024) VEDA_HIP_TRY(hipFuncSetAttribute((const void*)kern, hipFuncAttributeMaxDynamicSharedMemorySize, kLds));
    hipLaunchKernelGGL(kern, dim3((unsigned)(a.items * a.c.kv_heads)), dim3(64 * kWaves), kLds, s, a);
    return launch_status("veda_packed_attn_fwd");
}

template <bool kBf16, int D, int RB> static veda_status launch_keys(const CacheAttnArgs& a, hipStream_t s) {
    constexpr int G = packed_groups<kBf16, D, RB>();
    if (!a.workers) {
        const int64_t groups = a.items * a.c.kv_heads;
        if (groups > 768) return launch_short<kBf16, D, RB, 2, 2>(a, s);
        return groups > 256 ? launch_short<kBf16, D, RB, 2, 4>(a, s) : launch_short<kBf16, D, RB, 2, 8>(a, s);
    }
    hipLaunchKernelGGL((packed_attn_share_kernel<kBf16, D, RB, G>), dim3((unsigned)a.workers), dim3(64), (PackedKeys<D, G>::kSlot), s, a);
    veda_status st = launch_status("veda_packed_attn_fwd");
    if (st != VEDA_OK) return st;
    // Rows are joined by a wave each, by 8 or by 16: as many as leave a few parts to each (16 caches of up to 16,000 keys, 4 rows of 32 heads on 4, 32 parts, by 8 / 16:
    // 40 / 45 us; 8 of up to 12,000, 2 rows of 12 heads, 21 parts, 26 / 27).
    typedef PackedKeys<D, G> P;
    const int64_t joins = (int64_t)a.c.rows * a.q_heads, parts = a.workers / a.c.kv_heads / a.c.seqs;      // of a row, about
    auto join = [&](auto kern, int64_t blocks, int threads) { hipLaunchKernelGGL(kern, dim3((unsigned)blocks), dim3((unsigned)threads), 0, s, a); };
    if (parts <= 8 || joins >= 1 << 22) join(cache_attn_join_parts_kernel<kBf16, D, RB, 1, P::kKeys, 8, P::kLeast>, (joins + 7) / 8, 512);
    else if (parts <= 64) join(cache_attn_join_parts_kernel<kBf16, D, RB, 8, P::kKeys, 4, P::kLeast>, joins, 512);
    else join(cache_attn_join_parts_kernel<kBf16, D, RB, 16, P::kKeys, 8, P::kLeast>, joins, 1024);
    return launch_status("veda_packed_attn_fwd");
}

template <bool kBf16, int D> static veda_status launch_keys_d(const CacheAttnArgs& a, hipStream_t s) {
    return a.part_rows == 16 ? launch_keys<kBf16, D, 1>(a, s) : launch_keys<kBf16, D, 2>(a, s);
}

veda_status launch_packed_attn_keys(const CacheAttnArgs& a, bool bf16, int d, hipStream_t s) {
    if (bf16) return d == 128 ? launch_keys_d<true, 128>(a, s) : launch_keys_d<true, 64>(a, s);
    return d == 128 ? launch_keys_d<false, 128>(a, s) : launch_keys_d<false, 64>(a, s);
}

}  // namespace veda
