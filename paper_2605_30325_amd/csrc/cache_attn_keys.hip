// Attention over the paged cache, few rows for each key head (single tokens and small chunks).
//
// O = sum_j p_j v_j / l with p_j = 2^(s_j - ref), l = sum_j p_j: sums over any keys can be formed apart and added once they are brought to a
// common reference.  Memory bounds it: every key and value is read once for at most 32 rows, so the work is to keep loads in flight on
// all compute units until the last of them is done.  The query heads that share a key head are put together as in cache_attn_rows.hip, 16
// rows to a product of 16 x 16 (K rows x query rows, and V channels x query rows): with 32 x 32 products, half or more of them padding, fp32
// tokens waited for the matrix cores (257 keys, 12 heads of 64: 18.6 us instead of 12.3).  A wave walks key tiles of its own, 16 or 32 keys, that direct
// loads put into its slots of LDS: no barrier in the loop, the compiler's waits only for what the wave itself has read.
//
// Long caches are shared out evenly.  The tiles of all sequences lie in one row of numbers; each of the waves that run at once takes one key
// head of an equal part of it, whatever sequences that cuts, and the heads of a part are neighbours: they read the same pages at the same
// time, which is worth a tenth of the bandwidth.  The pieces of a cut sequence go to the workspace as unfinished sums, at most two a wave,
// and cache_attn_join_parts_kernel puts them together.  d = 128, bf16, 8 key heads: 64 caches of 8192 keys 353-371 us from box to box (5.8-6.1 TB/s); 64 of 1..8192
// keys 192-196 us (5.5 TB/s; a workgroup for each sequence and head waits for the longest: 208-235); one of 131,101 keys 105 us (5.1 TB/s), of
// 400,001 283 us (5.8).
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

template <bool kBf16, int D, int RB> struct KeysRow {
    f32x4v o[RB][D / 16];
    bf16x8 qb[RB][kBf16 ? D / 32 : 1];
    float qf[RB][kBf16 ? 1 : D / 4];
    float ref[RB], sub[RB], l[RB];   // reference of the exponentials (log2 units), 0 or -ref, this lane's sum
    int lo[RB], hi[RB];              // visible keys
};

// bf16: operand of V for channels 16 c.. of 32 keys, by transposing reads: elements 0-3 are keys 4 g + e, 4-7 keys 16 + 4 g + e.
template <int D> __device__ __forceinline__ bf16x8 keys_v(uint32_t v, int c) {
    const uint32_t at = v ^ (uint32_t)(c << 5);
    const bf16x4 x = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds_bf16x4_p)(uintptr_t)at);
    const bf16x4 y = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds_bf16x4_p)(uintptr_t)(at + 16 * (D * 2)));
    return __builtin_shufflevector(x, y, 0, 1, 2, 3, 4, 5, 6, 7);
}
// f32: V for channels 16 c.., key 16 b + 4 g + i.
template <int D> __device__ __forceinline__ float keys_v32(uint32_t v, int c, int b, int i) {
    return *(lds_f32_ptr)(uintptr_t)((v ^ (uint32_t)(c << 6)) + (16 * b + i) * (D * 4));
}

// bf16: a weight goes into its product in two parts, 2^-15 of it off at most (one part: 2^-8, which is as much as the results' own rounding).  The
// matrix cores have the time: us with one / two parts, d = 128: ragged single tokens of 64 streams 193.7 / 193.4, one of a cache of 131,101 105.6 /
// 105.8, 64 of 501 keys 23.9 / 24.2, 512 of 101 51.0 / 51.9; 32 rows of 16 caches of 4100 keys, the dearest, 57.2 / 60.8.
// The first part is the largest value below the weight, so that the rest of a weight above 0 is above 0 too: neither part's product with an
// infinite value is NaN.
__device__ __forceinline__ __bf16 keys_part(float p) {
    return __builtin_bit_cast(__bf16, (uint16_t)(__builtin_elementwise_sub_sat(__builtin_bit_cast(uint32_t, p), 1u) >> 16));
}

// A tile of keys from key0 on for one wave.  full: every row sees all of them.  exists: bit b = keys 16 b .. 16 b + 15 exist.
template <bool kBf16, int D, int RB>
__device__ __forceinline__ void keys_tile(const CacheAttnArgs& a, KeysRow<kBf16, D, RB>& st, uint32_t k, uint32_t v, int key0, uint32_t exists,
                                          bool full, int g) {
    constexpr int kRowB = KeysTile<kBf16, D>::kRowB, C = D / 16, B = KeysTile<kBf16, D>::kGroups;
    f32x4v s[RB][B];
#pragma unroll
    for (int rb = 0; rb < RB; ++rb)
#pragma unroll
        for (int b = 0; b < B; ++b) s[rb][b] = f32x4v{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int b = 0; b < B; ++b) {
        if constexpr (kBf16) {
#pragma unroll
            for (int t = 0; t < D / 32; ++t) {
                const bf16x8 x = *(lds_bf16x8_p)(uintptr_t)((k ^ (uint32_t)(t << 6)) + b * 16 * kRowB);
#pragma unroll
                for (int rb = 0; rb < RB; ++rb) s[rb][b] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(x, st.qb[rb][t], s[rb][b], 0, 0, 0);
            }
        } else {
#pragma unroll
            for (int u = 0; u < D / 16; ++u) {
                const f32x4v x = *(lds_f32x4_ptr)(uintptr_t)((k ^ (uint32_t)(u << 6)) + b * 16 * kRowB);
#pragma unroll
                for (int e = 0; e < 4; ++e)
#pragma unroll
                    for (int rb = 0; rb < RB; ++rb) s[rb][b] = __builtin_amdgcn_mfma_f32_16x16x4f32(x[e], st.qf[rb][4 * u + e], s[rb][b], 0, 0, 0);
            }
        }
    }
    auto seen = [&](int rb, int b, int i) __attribute__((always_inline)) {
        const int key = key0 + 16 * b + 4 * g + i;
        return key < st.hi[rb] && (key >= st.lo[rb] || key < a.sinks) && ((exists >> b) & 1u);
    };
    float mx[RB];
    bool grown = false;
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) {
        if (!full) {
#pragma unroll
            for (int b = 0; b < B; ++b)
#pragma unroll
                for (int i = 0; i < 4; ++i) s[rb][b][i] = seen(rb, b, i) ? s[rb][b][i] : -INFINITY;
        }
        float m = s[rb][0][0];
#pragma unroll
        for (int b = 0; b < B; ++b)
#pragma unroll
            for (int i = 0; i < 4; ++i) m = fmaxf(m, s[rb][b][i]);
        mx[rb] = m * a.scale_log2;
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
    bf16x8 p[kBf16 ? RB : 1], rest[kBf16 ? RB : 1];
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) {
        float sum = 0.0f;
#pragma unroll
        for (int b = 0; b < B; ++b)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                s[rb][b][i] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[rb][b][i], a.scale_log2, st.sub[rb]));
                sum += s[rb][b][i];
                if constexpr (kBf16) {
                    p[rb][4 * b + i] = keys_part(s[rb][b][i]);
                    rest[rb][4 * b + i] = (__bf16)(s[rb][b][i] - (float)p[rb][4 * b + i]);
                }
            }
        st.l[rb] += sum;
    }
    // A product with zeros is not zero where a value is infinite or NaN: such values reach only the rows that see them.
    bool plain = true;
    if (!full) {
        f32x4v z = {0.0f, 0.0f, 0.0f, 0.0f};
        if constexpr (kBf16) {
            bf16x8 zero;
#pragma unroll
            for (int e = 0; e < 8; ++e) zero[e] = (__bf16)0.0f;
#pragma unroll
            for (int c = 0; c < C; ++c) z = __builtin_amdgcn_mfma_f32_16x16x32_bf16(keys_v<D>(v, c), zero, z, 0, 0, 0);
        } else {
#pragma unroll
            for (int b = 0; b < B; ++b)
#pragma unroll
                for (int i = 0; i < 4; ++i)
#pragma unroll
                    for (int c = 0; c < C; ++c) z = __builtin_amdgcn_mfma_f32_16x16x4f32(keys_v32<D>(v, c, b, i), 0.0f, z, 0, 0, 0);
        }
        plain = !__any(z[0] + z[1] + z[2] + z[3] != 0.0f);   // NaN != 0
    }
    if (plain) {
        if constexpr (kBf16) {
#pragma unroll
            for (int c = 0; c < C; c += 2) {   // two at a time, so that a sum's next product is not the one right behind it
                const bf16x8 x[2] = {keys_v<D>(v, c), keys_v<D>(v, c + 1)};
#pragma unroll
                for (int j = 0; j < 4 * RB; ++j) {
                    const int rb = j / 2 % RB, i = c + j % 2;
                    st.o[rb][i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(x[j % 2], j < 2 * RB ? p[rb] : rest[rb], st.o[rb][i], 0, 0, 0);
                }
            }
        } else {
#pragma unroll
            for (int b = 0; b < B; ++b)
#pragma unroll
                for (int i = 0; i < 4; ++i)
#pragma unroll
                    for (int c = 0; c < C; ++c) {
                        const float x = keys_v32<D>(v, c, b, i);
#pragma unroll
                        for (int rb = 0; rb < RB; ++rb) st.o[rb][c] = __builtin_amdgcn_mfma_f32_16x16x4f32(x, s[rb][b][i], st.o[rb][c], 0, 0, 0);
                    }
        }
    } else {
#pragma unroll
        for (int c = 0; c < C; ++c) {
            f32x4v code[RB];
#pragma unroll
            for (int rb = 0; rb < RB; ++rb) code[rb] = f32x4v{0.0f, 0.0f, 0.0f, 0.0f};
            if constexpr (kBf16) {
                bf16x8 x = keys_v<D>(v, c), y;
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    y[e] = (__bf16)attn_code((float)x[e]);
                    x[e] = (float)y[e] == 0.0f ? x[e] : (__bf16)0.0f;
                }
#pragma unroll
                for (int rb = 0; rb < RB; ++rb) {
                    bf16x8 on;
#pragma unroll
                    for (int e = 0; e < 8; ++e) on[e] = (__bf16)attn_times((float)p[rb][e], seen(rb, e / 4, e % 4));
                    st.o[rb][c] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(x, p[rb], st.o[rb][c], 0, 0, 0);
                    st.o[rb][c] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(x, rest[rb], st.o[rb][c], 0, 0, 0);
                    code[rb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(y, on, code[rb], 0, 0, 0);
                }
            } else {
#pragma unroll
                for (int b = 0; b < B; ++b)
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const float x = keys_v32<D>(v, c, b, i), y = attn_code(x);
#pragma unroll
                        for (int rb = 0; rb < RB; ++rb) {
                            st.o[rb][c] = __builtin_amdgcn_mfma_f32_16x16x4f32(y == 0.0f ? x : 0.0f, s[rb][b][i], st.o[rb][c], 0, 0, 0);
                            code[rb] = __builtin_amdgcn_mfma_f32_16x16x4f32(y, attn_times(s[rb][b][i], seen(rb, b, i)), code[rb], 0, 0, 0);
                        }
                    }
            }
#pragma unroll
            for (int rb = 0; rb < RB; ++rb)
#pragma unroll
                for (int i = 0; i < 4; ++i) st.o[rb][c][i] += attn_decode(code[rb][i]);
            __builtin_amdgcn_sched_barrier(0);
        }
    }
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

// What a lane adds to addresses: of the loads (lane i of a load lands at byte 16 i of its KB, so the swizzle is applied to what it
// fetches) and of the operands.
template <bool kBf16, int D> struct KeysLane {
    typedef KeysTile<kBf16, D> T;
    uint32_t k_off, v_off, k_at, v_at;
    int l15, g;
    __device__ __forceinline__ explicit KeysLane(int lane) : l15(lane & 15), g(lane >> 4) {
        const int row = lane / T::kChunks, c = lane % T::kChunks;
        k_off = (uint32_t)(row * T::kRowB + ((c ^ T::k_swizzle(row)) << 4));
        v_off = (uint32_t)(row * T::kRowB + ((c ^ T::v_swizzle(row)) << 4));
        k_at = (uint32_t)(l15 * T::kRowB + ((g ^ T::k_swizzle(l15)) << 4));
        if constexpr (kBf16) {
            // transposing read: lane i of 16 names channels 4 (i % 4) ..+3 of key i / 4 and gets channel i of the four keys
            const int key = 4 * g + (l15 >> 2);
            v_at = (uint32_t)(key * T::kRowB + ((((l15 & 3) >> 1) ^ T::v_swizzle(key)) << 4) + 8 * (l15 & 1));
        } else {
            v_at = (uint32_t)(4 * g * T::kRowB + 4 * l15 + (g << 6));
        }
        v_at += T::kKeys * T::kRowB;
    }
    // Asks for a tile: from[b] is where its 16 keys number b begin in either pool.
    __device__ __forceinline__ void load(const CacheArgs& c, const int64_t (&from)[T::kGroups], uint32_t lds) const {
#pragma unroll
        for (int sg = 0; sg < T::kSegs; ++sg) {
            const int row = sg * T::kSegRows;
            const int64_t at = from[row / 16] + row % 16 * T::kRowB;
            uint32_t k[T::kSegLoads], v[T::kSegLoads];
#pragma unroll
            for (int j = 0; j < T::kSegLoads; ++j) {
                k[j] = k_off ^ T::k_step(j);
                v[j] = v_off ^ T::v_step(sg, j);
            }
            dma16_group_to_lds<T::kSegLoads>(lds + row * T::kRowB, c.k + at, k);
            dma16_group_to_lds<T::kSegLoads>(lds + (T::kKeys + row) * T::kRowB, c.v + at, v);
        }
    }
};

// The rows of a block: what they see and ask for, and no sums yet.
struct KeysSeen { int lo, hi, lo_all, hi_all; };   // some row sees keys from lo and below hi, every row those from lo_all and below hi_all
template <bool kBf16, int D, int RB>
__device__ __forceinline__ KeysSeen keys_rows(const CacheAttnArgs& a, KeysRow<kBf16, D, RB>& st, const SeqRows& sr, int n, int head, int r0, int r_end,
                                              int l15, int g) {
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) {
        const int r = min(r0 + 16 * rb + l15, r_end - 1);
        const Seen see = seen_by(a, sr, n, r);
        st.lo[rb] = see.lo;
        st.hi[rb] = see.hi;
        const char* q = a.q + (int64_t)(sr.first + r / a.group) * a.sq_n + (int64_t)(head * a.group + r % a.group) * a.sq_h;
        if constexpr (kBf16) {
#pragma unroll
            for (int t = 0; t < D / 32; ++t) st.qb[rb][t] = *reinterpret_cast<const bf16x8*>(q + 64 * t + 16 * g);
        } else {
#pragma unroll
            for (int u = 0; u < D / 16; ++u) {
                const f32x4v x = *reinterpret_cast<const f32x4v*>(q + 64 * u + 16 * g);
#pragma unroll
                for (int e = 0; e < 4; ++e) st.qf[rb][4 * u + e] = x[e];
            }
        }
#pragma unroll
        for (int c = 0; c < D / 16; ++c) st.o[rb][c] = f32x4v{0.0f, 0.0f, 0.0f, 0.0f};
        st.ref[rb] = -INFINITY;
        st.sub[rb] = st.l[rb] = 0.0f;
    }
    return {__builtin_amdgcn_readlane(st.lo[0], 0), __builtin_amdgcn_readlane(st.hi[RB - 1], 15), __builtin_amdgcn_readlane(st.lo[RB - 1], 15),
            __builtin_amdgcn_readlane(st.hi[0], 0)};
}

// Where 16 keys from token `tok` on begin in the pools (head_b: the head's rows in a page), and whether they exist.
__device__ __forceinline__ bool keys_from(const CacheArgs& c, const int32_t* table, int len, int64_t head_b, int row_b, int tok, int64_t& from) {
    const int id = tok < len ? table[tok >> c.log_page] : -1;
    const bool ok = id >= 0 && id < c.pages;
    from = ok ? id * c.page_b + head_b + (int64_t)(tok & ((1 << c.log_page) - 1)) * row_b : head_b;   // any place in the pool will do
    return ok;
}

template <bool kBf16, int D, int RB>
__device__ __forceinline__ void keys_step(const CacheAttnArgs& a, KeysRow<kBf16, D, RB>& st, const KeysSeen& see, const KeysLane<kBf16, D>& ln, uint32_t lds,
                                          int key0, uint32_t exists) {
    typedef KeysTile<kBf16, D> T;
    const int end = key0 + T::kKeys;
    if (key0 >= see.hi || (end <= see.lo && key0 >= a.sinks) || exists == 0) return;
    const bool full = end <= see.hi_all && (key0 >= see.lo_all || end <= a.sinks) && exists == (1u << T::kGroups) - 1;
    keys_tile<kBf16, D, RB>(a, st, lds + ln.k_at, lds + ln.v_at, key0, exists, full, ln.g);
}

// 64-bit value of another lane, the same for all.
__device__ __forceinline__ int64_t lane_value(int64_t x, int lane) {
    return (int64_t)((uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(uint64_t)x, lane) |
                     (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)((uint64_t)x >> 32), lane) << 32);
}

// Short caches: a workgroup for each (block of rows, key head), whose waves take its tiles in turn.  With few workgroups latency counts:
// eight waves (32 fp32 rows of 128: four, or their registers do not do) with a slot each, so that all of a cache of 256 keys, half of one of 512, is asked for at once.  With
// more than there are compute units two waves with two slots, so that workgroups start while others end.  Two waves / eight, us: one
// fp32 token over 257 keys, 12 heads of 64, 12.3 / 9.1; bf16, d = 128, 64 workgroups of 501 keys 12.4 / 10.4, 512 of 401 21.3 / 25, 4096
// of 101 54 / 88; fp32, d = 64, 768 of 401 44 / 40.
template <bool kBf16, int D, int RB, bool kMany> struct KeysGroup {
    static constexpr int kWaves = kMany ? 2 : kBf16 || D == 64 || RB == 1 ? 8 : 4, kSlots = kMany ? 2 : 1;
};
template <bool kBf16, int D, int RB, bool kMany>
__global__ __launch_bounds__((64 * KeysGroup<kBf16, D, RB, kMany>::kWaves)) void cache_attn_keys_kernel(CacheAttnArgs a) {
    typedef KeysTile<kBf16, D> T;
    constexpr int kRows = 16 * RB, kEs = kBf16 ? 2 : 4, kWaves = KeysGroup<kBf16, D, RB, kMany>::kWaves, kSlots = KeysGroup<kBf16, D, RB, kMany>::kSlots;
    extern __shared__ __align__(1024) char smem[];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const KeysLane<kBf16, D> ln(lane);
    const uint32_t lds = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)smem + wave * kSlots * T::kSlot;
    RowBlock block;
    if (!block_of(a.c, a.group, kRows, a.per_seq, blockIdx.x / a.c.kv_heads, block)) return;
    const int head = blockIdx.x % a.c.kv_heads, r0 = block.block * kRows;
    const SeqRows sr = block.rows;
    const int n = min(sr.n, a.c.max_new), r_end = min(n * a.group, r0 + kRows);
    const AttnTiles tiles = tiles_seen(a, sr, n, r0, r_end - 1, T::kKeys);
    const int32_t* table = a.c.table + block.seq * a.c.table_stride;
    const int64_t head_b = (int64_t)head * T::kRowB << a.c.log_page;

    // Places of the wave's next 64 tiles, one tile a lane: looked up together, so that no step waits for the table.
    int64_t from[T::kGroups] = {};
    uint32_t there = 0;
    auto look_up = [&](int t) {
        const int mine = t + lane * kWaves;
        there = 0;
#pragma unroll
        for (int b = 0; b < T::kGroups; ++b)
            there |= (keys_from(a.c, table, mine < tiles.count ? sr.len : 0, head_b, T::kRowB, tiles.at(mine) + 16 * b, from[b]) ? 1u : 0u) << b;
    };
    auto load = [&](int at, int slot) {
        int64_t f[T::kGroups];
#pragma unroll
        for (int b = 0; b < T::kGroups; ++b) f[b] = lane_value(from[b], at);
        ln.load(a.c, f, lds + slot * T::kSlot);
    };
    int slot = 0, at = 0;
    if (wave < tiles.count) {
        look_up(wave);
        load(0, 0);
    }
    KeysRow<kBf16, D, RB> st;
    const KeysSeen see = keys_rows<kBf16, D, RB>(a, st, sr, n, head, r0, r_end, ln.l15, ln.g);
    for (int t = wave; t < tiles.count; t += kWaves) {
        const uint32_t exists = (uint32_t)__builtin_amdgcn_readlane((int)there, at);
        const bool more = t + kWaves < tiles.count;
        if (++at == 64 && more) {
            look_up(t + kWaves);
            at = 0;
        }
        if (kSlots == 2 && more) {
            __builtin_amdgcn_s_waitcnt(0xc07f);   // lgkmcnt(0): the other slot has been read
            load(at, slot ^ 1);
            wait_vmcnt<T::kLoads>();
        } else {
            wait_vmcnt<0>();
        }
        asm volatile("" ::: "memory");
        keys_step<kBf16, D, RB>(a, st, see, ln, lds + slot * T::kSlot, tiles.at(t), exists);
        if (kSlots == 1 && more) {
            __builtin_amdgcn_s_waitcnt(0xc07f);
            load(at, 0);
        }
        if (kSlots == 2) slot ^= 1;
    }

    // Sums of the waves, put together row by row.  A lane holds channels 16 c + 4 g + 0..3 of its row.
    __syncthreads();
    float* ml = reinterpret_cast<float*>(smem + kWaves * kRows * T::kOutRowB);   // [wave][row][2]
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) {
        const int row = wave * kRows + 16 * rb + ln.l15;
        const float l = keys_sum(st.l[rb]);
#pragma unroll
        for (int c = 0; c < D / 16; ++c) *reinterpret_cast<f32x4v*>(smem + row * T::kOutRowB + (16 * c + 4 * ln.g) * 4) = st.o[rb][c];
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
            o += f * *reinterpret_cast<const f32x4v*>(smem + (w * kRows + rr) * T::kOutRowB + ch * 4);
        }
        const int64_t token = sr.first + row / a.group;
        const int qh = head * a.group + row % a.group;
        keys_store<kBf16>(a.out + token * a.so_n + (int64_t)qh * a.so_h + ch * kEs, o * attn_inverse(a, block.seq, sr, row, l));
        if (a.lse && ch == 0) a.lse[(int64_t)qh * a.c.rows + token] = attn_lse(ref, l);
    }
}

// Long caches: every wave is a workgroup and takes one key head of an equal part [now, end) of the common row of tiles, sequence by
// sequence.  Loads run kDepth - 1 tiles ahead across their ends, so a change of sequence costs the new rows' loads and no more.  (Two slots
// instead of three: 64 even caches of 8192 keys 376 us instead of 353; a workgroup of several waves that stops at every end: 82 us instead
// of 53 for ten ragged caches of 12 heads.)
template <bool kBf16, int D, int RB> __global__ __launch_bounds__(64) void cache_attn_share_kernel(CacheAttnArgs a) {
    typedef KeysTile<kBf16, D> T;
    constexpr int kRows = 16 * RB, kEs = kBf16 ? 2 : 4;
    extern __shared__ __align__(1024) char smem[];
    const int lane = threadIdx.x;
    const KeysLane<kBf16, D> ln(lane);
    const uint32_t lds = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)smem;
    const KeysCount count(a, T::kKeys);
    const TileShare share(count.total, a.workers / a.c.kv_heads, kShareTiles);
    const int head = blockIdx.x % a.c.kv_heads, mine = blockIdx.x / a.c.kv_heads;
    if (mine >= share.parts || share.total == 0) return;
    int now = share.begin(mine);
    const int end = share.begin(mine + 1);
    const int64_t head_b = (int64_t)head * T::kRowB << a.c.log_page;

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
            p.tiles = tiles_seen(a, p.sr, n, 0, n * a.group - 1, T::kKeys);
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
    // Places of the next 64 tiles, one tile a lane, whichever sequences they belong to.
    int64_t from[T::kGroups];
#pragma unroll
    for (int b = 0; b < T::kGroups; ++b) from[b] = head_b;
    uint32_t there = 0;
    auto look_up = [&](int x) {
        const int at = x + lane;
        there = 0;
        while (ahead.each) {
            const int last = ahead.first + ahead.each, t = at - ahead.first;
            if (t >= 0 && at < last && at < end) {
                const int32_t* table = a.c.table + ahead.seq * a.c.table_stride;
#pragma unroll
                for (int b = 0; b < T::kGroups; ++b)
                    there |= (keys_from(a.c, table, t < ahead.tiles.count ? ahead.sr.len : 0, head_b, T::kRowB, ahead.tiles.at(t) + 16 * b, from[b]) ? 1u : 0u) << b;
            }
            if (last >= min(x + 64, end)) break;
            enter(ahead, ahead.seq + 1, last);
        }
    };
    // Tiles asked for, the last of them number `at` - 1 of those looked up; ex: which keys of tiles now, now + 1, .. exist.
    int asked = now, at = 64, ask_slot = 0, slot = 0;
    uint32_t ex[T::kDepth];
    auto ask = [&](uint32_t& e) __attribute__((always_inline)) {
        if (asked >= end) return;
        if (at == 64) {
            look_up(asked);
            at = 0;
        }
        int64_t f[T::kGroups];
#pragma unroll
        for (int b = 0; b < T::kGroups; ++b) f[b] = lane_value(from[b], at);
        e = (uint32_t)__builtin_amdgcn_readlane((int)there, at);
        ln.load(a.c, f, lds + ask_slot * T::kSlot);
        ask_slot = ask_slot + 1 == T::kDepth ? 0 : ask_slot + 1;
        ++at;
        ++asked;
    };
#pragma unroll
    for (int j = 0; j + 1 < T::kDepth; ++j) ask(ex[j]);
    while (now < end && here.each) {
        const SeqRows sr = here.sr;
        const int n = min(sr.n, a.c.max_new), rows = n * a.group;
        const int t_beg = now - here.first, stop = min(end, here.first + here.each);
        KeysRow<kBf16, D, RB> st;
        const KeysSeen see = keys_rows<kBf16, D, RB>(a, st, sr, n, head, 0, rows, ln.l15, ln.g);
        for (; now < stop; ++now) {
            __builtin_amdgcn_s_waitcnt(0xc07f);   // lgkmcnt(0): the slot to fill has been read
            ask(ex[T::kDepth - 1]);
            if (asked - now == 3) wait_vmcnt<2 * T::kLoads>();
            else if (asked - now == 2) wait_vmcnt<T::kLoads>();
            else wait_vmcnt<0>();
            asm volatile("" ::: "memory");
            keys_step<kBf16, D, RB>(a, st, see, ln, lds + slot * T::kSlot, here.tiles.at(now - here.first), ex[0]);
            slot = slot + 1 == T::kDepth ? 0 : slot + 1;
#pragma unroll
            for (int j = 0; j + 1 < T::kDepth; ++j) ex[j] = ex[j + 1];
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
                for (int c = 0; c < D / 16; ++c) *reinterpret_cast<f32x4v*>(po + 16 * c) = st.o[rb][c];
                if (ln.g == 0) *reinterpret_cast<f32x2v*>(a.part + (int64_t)2 * a.workers * kRows * D + (part * kRows + row) * 2) = f32x2v{st.ref[rb], l};
                continue;
            }
            const int64_t token = sr.first + row / a.group;
            const int qh = head * a.group + row % a.group;
            char* dst = a.out + token * a.so_n + (int64_t)qh * a.so_h + 4 * ln.g * kEs;
            const float inv = attn_inverse(a, here.seq, sr, row, l);
#pragma unroll
            for (int c = 0; c < D / 16; ++c) keys_store<kBf16>(dst + 16 * c * kEs, st.o[rb][c] * inv);
            if (a.lse && ln.g == 0) a.lse[(int64_t)qh * a.c.rows + token] = attn_lse(st.ref[rb], l);
        }
        if (now == here.first + here.each) enter(here, here.seq + 1, now);
    }
    wait_vmcnt<0>();
}

// Puts the unfinished sums of a (row, query head) together; rows that one workgroup had whole have none.  W waves for each: one
// where there are about as many sequences as parts, eight (four loads in flight each) for few long sequences, cut into many.
template <bool kBf16, int D, int RB, int W> __global__ __launch_bounds__(512) void cache_attn_join_parts_kernel(CacheAttnArgs a) {
    constexpr int kRows = 16 * RB, V = D / 64;
    __shared__ float sums[W][D + 2];
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, w = wave % W;
    const int64_t item = (int64_t)blockIdx.x * (8 / W) + wave / W;
    const bool is_row = item < (int64_t)a.c.rows * a.q_heads;
    const int token = is_row ? (int)(item / a.q_heads) : -1, qh = (int)(item % a.q_heads);
    // the row's sequence, and its tiles
    int first = 0, each = 0, row = 0, total = 0, seq = 0;
    for (int s0 = 0; s0 < a.c.seqs; s0 += 64) {
        const int s = s0 + lane;
        int mine = 0, i = -1;
        if (s < a.c.seqs) {
            mine = keys_tiles_of(a, s, KeysTile<kBf16, D>::kKeys);
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
    const TileShare share(total, a.workers / a.c.kv_heads, kShareTiles);
    const int w0 = each ? share.owner(first) : 0, n = each ? share.owner(first + each - 1) - w0 + 1 : 1;
    if (n == 1) return;   // one workgroup had it all (with W = 8 the same for all waves)
    const float2* ml = reinterpret_cast<const float2*>(a.part + (int64_t)2 * a.workers * kRows * D);
    auto part_row = [&](int j) { return (2 * ((int64_t)(w0 + j) * a.c.kv_heads + qh / a.group) + (j == 0 ? 1 : 0)) * kRows + row; };
    float2 m[4];
    float x[4][V];
    auto get = [&](int j0) {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int64_t at = part_row(min(j0 + W * j, n - 1));
            m[j] = ml[at];
#pragma unroll
            for (int c = 0; c < V; ++c) x[j][c] = a.part[at * D + V * lane + c];
        }
    };
    get(w);   // on their way while the common reference is found
    float ref = -INFINITY;
    for (int j = lane; j < n; j += 64) ref = fmaxf(ref, ml[part_row(j)].x);
#pragma unroll
    for (int x = 32; x >= 1; x >>= 1) ref = fmaxf(ref, __shfl_xor(ref, x));
    float l = 0.0f, o[V];
#pragma unroll
    for (int c = 0; c < V; ++c) o[c] = 0.0f;
    for (int j0 = w; j0 < n; j0 += 4 * W) {
        if (j0 != w) get(j0);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
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

template <bool kBf16, int D> static constexpr int keys_slots() { return KeysTile<kBf16, D>::kDepth * KeysTile<kBf16, D>::kSlot; }
int attn_keys_workers(bool bf16, int d) {
    const int slots = bf16 ? (d == 128 ? keys_slots<true, 128>() : keys_slots<true, 64>()) : (d == 128 ? keys_slots<false, 128>() : keys_slots<false, 64>());
    // Waves to a compute unit: as many as its LDS has slots for, but no more than four, and not to the last byte (five waves of 32 KB, or
    // four of 48, did not run at once: a quarter of the work came behind the rest).
    const int fit = 159 * 1024 / slots;
    return 256 * (fit < 4 ? fit : 4);
}

template <bool kBf16, int D, int RB, bool kMany> static veda_status launch_short(const CacheAttnArgs& a, hipStream_t s) {
    typedef KeysGroup<kBf16, D, RB, kMany> G;
    constexpr int kSums = G::kWaves * 16 * RB * (KeysTile<kBf16, D>::kOutRowB + 8), kTiles = G::kWaves * G::kSlots * KeysTile<kBf16, D>::kSlot;
    constexpr int kLds = kTiles > kSums ? kTiles : kSums;
    static_assert(kLds <= 160 * 1024, "what a compute unit has");
    auto kern = cache_attn_keys_kernel<kBf16, D, RB, kMany>;
    if (kLds > 64 * 1024) VEDA_HIP_TRY(hipFuncSetAttribute((const void*)kern, hipFuncAttributeMaxDynamicSharedMemorySize, kLds));
    hipLaunchKernelGGL(kern, dim3((unsigned)(a.items * a.c.kv_heads)), dim3(64 * G::kWaves), kLds, s, a);
    return launch_status("veda_cache_attn_fwd");
}

template <bool kBf16, int D, int RB> static veda_status launch_keys(const CacheAttnArgs& a, hipStream_t s) {
    static_assert(keys_slots<kBf16, D>() <= 64 * 1024, "what a launch may have without asking");
    if (!a.workers) {
        if constexpr (kBf16)
            if (a.items * a.c.kv_heads > 256) return launch_short<kBf16, D, RB, true>(a, s);
        return launch_short<kBf16, D, RB, false>(a, s);
    }
    hipLaunchKernelGGL((cache_attn_share_kernel<kBf16, D, RB>), dim3((unsigned)a.workers), dim3(64), (keys_slots<kBf16, D>()), s, a);
    veda_status st = launch_status("veda_cache_attn_fwd");
    if (st != VEDA_OK) return st;
    const int64_t joins = (int64_t)a.c.rows * a.q_heads;
    if (a.workers / a.c.kv_heads > 8 * a.c.seqs && joins < 1 << 23) hipLaunchKernelGGL((cache_attn_join_parts_kernel<kBf16, D, RB, 8>), dim3((unsigned)joins), dim3(512), 0, s, a);
    else hipLaunchKernelGGL((cache_attn_join_parts_kernel<kBf16, D, RB, 1>), dim3((unsigned)((joins + 7) / 8)), dim3(512), 0, s, a);
    return launch_status("veda_cache_attn_fwd");
}

template <bool kBf16, int D> static veda_status launch_keys_d(const CacheAttnArgs& a, hipStream_t s) {
    return a.part_rows == 16 ? launch_keys<kBf16, D, 1>(a, s) : launch_keys<kBf16, D, 2>(a, s);
}

veda_status launch_cache_attn_keys(const CacheAttnArgs& a, bool bf16, int d, hipStream_t s) {
    if (bf16) return d == 128 ? launch_keys_d<true, 128>(a, s) : launch_keys_d<true, 64>(a, s);
    return d == 128 ? launch_keys_d<false, 128>(a, s) : launch_keys_d<false, 64>(a, s);
}

}  // namespace veda
