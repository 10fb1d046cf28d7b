// Attention over the paged cache, blocks of many rows.
//
// The query heads that share a key head are put together: row r of a (sequence, key head) is query head r % G of token r / G,
// so a key that is loaded once serves G heads.  Scores are formed transposed (S^T = K Q^T, O^T = V^T P^T): a lane owns one row,
// its accumulators run over keys, the running maximum and sum of the softmax stay in registers, and P^T is the second product's operand
// as it stands.  The reference of the exponentials follows the maximum only when that has outgrown it by 2^8: any reference gives the same
// quotient.  Logits are scaled in fp32 on their way into the exponential, so Q is not rounded again; P is rounded to bf16 for its product
// (half a step, 2^-8 of each weight, and independent from key to key; a second part, as few rows have it, would be half as many matrix
// instructions again where these bound the kernel), l sums the weights before that.
//
// A workgroup takes 128 rows, 32 a wave; its four waves load a tile of keys together (straight into LDS, one tile ahead, 64 KB for two
// tiles of 64 keys at d = 128, so two workgroups to a compute unit) and each attends to all of it.  K and V lie token by token as they
// were appended: rows of K are operands as they stand, V is transposed by gfx950's transposing LDS reads.
//
// What bounds it: the matrix cores, and the power they draw.  4680 rows x 12 heads on 34,320 keys, d = 128, bf16: 0.90-0.95 ms from box to box =
// 1.04-1.10 PFLOP/s (a large matrix product reaches 1.22); matrix pipes 55 % busy at 1.9 GHz, 63 % on the compute units that hold two workgroups
// (444 on 512 places).  Prompts of 1..4096 tokens, G = 4, window 1024: 0.30-0.33 ms = 0.79-0.87 PFLOP/s; about 15 tiles of 64 keys that all rows see, three that
// some do, and as long again as two of them for the set-up and the results.  fp32 (v_mfma_f32_32x32x2_f32): 2464 rows x 12 heads on 2000 keys, causal, 0.35 ms,
// matrix pipes 73 % busy, 102 TFLOP/s on visible keys of the 154 that a large product reaches.
#include "cache_attn.h"
#include "store.h"

namespace veda {

template <bool kBf16, int D> struct AttnTile {
    static constexpr int kRowB = D * (kBf16 ? 2 : 4), kChunks = kRowB / 16;
    static constexpr int kSegRows = kBf16 ? 16 : 8;               // rows of a group of loads: never across a page's end
    static constexpr int kSegLoads = kSegRows * kRowB / 1024;     // 1 KB each
    // 16-byte chunk c of row r lies at chunk c ^ swizzle: operand reads of a wave then fall into different banks.
    __device__ static int k_swizzle(int r) { return kBf16 ? (D == 128 ? r & 15 : (r >> 1) & 7) : r & 7; }
    __device__ static int v_swizzle(int r) { return kBf16 ? (D == 128 ? (r & 3) << 2 : ((r >> 1) & 1) << 2) : ((r >> 2) & 1) << 3; }
    // What the swizzles of load j of a segment (1024 / kRowB rows each) have on top of load 0's, as address bits.
    __device__ static constexpr uint32_t k_step(int j) { return (uint32_t)j << (kBf16 || D == 64 ? 6 : 5); }
    __device__ static constexpr uint32_t v_step(int j) { return kBf16 ? 0u : (uint32_t)(D == 64 ? j : j >> 1) << 7; }
};

template <bool kBf16, int D> struct AttnRow {
    f32x16 o[D / 32];
    bf16x8 qb[kBf16 ? D / 16 : 1];
    float qf[kBf16 ? 1 : D / 2];
    float ref, sub, l;   // reference of the exponentials (log2 units), 0 or -ref, this half's sum
    int lo, hi;          // visible keys
};

// Scores of 32 keys whose K rows lie at LDS address `k` (+ the lane's part).
template <bool kBf16, int D> __device__ __forceinline__ f32x16 attn_scores(const AttnRow<kBf16, D>& st, uint32_t k) {
    f32x16 s;
#pragma unroll
    for (int i = 0; i < 16; ++i) s[i] = 0.0f;
    if constexpr (kBf16) {
#pragma unroll
        for (int t = 0; t < D / 16; ++t)
            s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(*(lds_bf16x8_p)(uintptr_t)(k ^ (uint32_t)(t << 5)), st.qb[t], s, 0, 0, 0);
    } else {
        // reads one group of products ahead, and no further: there are no registers for more
        f32x4v x = *(lds_f32x4_ptr)(uintptr_t)k;
#pragma unroll
        for (int u = 0; u < D / 8; ++u) {
            f32x4v next = x;
            if (u + 1 < D / 8) next = *(lds_f32x4_ptr)(uintptr_t)(k ^ (uint32_t)((u + 1) << 5));
#pragma unroll
            for (int e = 0; e < 4; ++e) s = __builtin_amdgcn_mfma_f32_32x32x2f32(x[e], st.qf[4 * u + e], s, 0, 0, 0);
            x = next;
            __builtin_amdgcn_sched_barrier(0);
        }
    }
    return s;
}

// Moves every row's reference up to its maximum mx (of this lane's half, log2 units) and rescales what was summed.
template <bool kBf16, int D> __device__ __forceinline__ void attn_move_ref(AttnRow<kBf16, D>& st, float mx) {
    const float ref = fmaxf(st.ref, max_with_other_half(mx));
    const float alpha = ref == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(st.ref - ref);
    st.ref = ref;
    st.sub = ref == -INFINITY ? 0.0f : -ref;
    st.l *= alpha;
#pragma unroll
    for (int nb = 0; nb < D / 32; ++nb)
#pragma unroll
        for (int i = 0; i < 16; ++i) st.o[nb][i] *= alpha;
}

// bf16: operand of V for channels 32 nb.. and key step kk (16 keys; the lane half's are 8 (e / 4) + 4 hh + e % 4), by transposing reads.
template <int D> __device__ __forceinline__ bf16x8 attn_v(uint32_t v, int kk, int nb) {
    const uint32_t at = (v ^ (uint32_t)(nb << 6)) + kk * 16 * (D * 2);
    const bf16x4 x = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds_bf16x4_p)(uintptr_t)at);
    const bf16x4 y = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds_bf16x4_p)(uintptr_t)(at + 8 * (D * 2)));
    return __builtin_shufflevector(x, y, 0, 1, 2, 3, 4, 5, 6, 7);
}

// Whether all values of 32 keys are finite: their product with zeros is zero exactly then.
template <int D> __device__ __forceinline__ bool attn_finite(uint32_t v) {
    bf16x8 zero;
    f32x16 z;
#pragma unroll
    for (int e = 0; e < 8; ++e) zero[e] = (__bf16)0.0f;
#pragma unroll
    for (int i = 0; i < 16; ++i) z[i] = 0.0f;
#pragma unroll
    for (int kk = 0; kk < 2; ++kk)
#pragma unroll
        for (int nb = 0; nb < D / 32; ++nb) {
            z = __builtin_amdgcn_mfma_f32_32x32x16_bf16(attn_v<D>(v, kk, nb), zero, z, 0, 0, 0);
            if (nb & 1) __builtin_amdgcn_sched_barrier(0);
        }
    float t = 0.0f;
#pragma unroll
    for (int i = 0; i < 16; ++i) t += z[i];
    return !__any(t != 0.0f);   // NaN != 0
}

// O^T += V^T P^T of 32 keys some of whose values are not finite: those reach the rows that see their keys (bit i: register i's).
template <int D> __device__ __forceinline__ void attn_careful(AttnRow<true, D>& st, uint32_t v, const bf16x8 (&p)[2], uint32_t seen) {
    constexpr int NB = D / 32;
    f32x16 o[NB];   // indexed as the loop goes, so it lies in memory: this path must not cost the others registers
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) o[nb] = st.o[nb];
#pragma unroll 1
    for (int nb = 0; nb < NB; ++nb) {
        f32x16 sum = o[nb], code;
#pragma unroll
        for (int i = 0; i < 16; ++i) code[i] = 0.0f;
#pragma unroll
        for (int kk = 0; kk < 2; ++kk) {
            bf16x8 x = attn_v<D>(v, kk, nb), y, on;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                y[e] = (__bf16)attn_code((float)x[e]);
                x[e] = (float)y[e] == 0.0f ? x[e] : (__bf16)0.0f;
                on[e] = (__bf16)attn_times((float)p[kk][e], (seen >> (8 * kk + e)) & 1u);
            }
            sum = __builtin_amdgcn_mfma_f32_32x32x16_bf16(x, p[kk], sum, 0, 0, 0);
            code = __builtin_amdgcn_mfma_f32_32x32x16_bf16(y, on, code, 0, 0, 0);
            __builtin_amdgcn_sched_barrier(0);
        }
#pragma unroll
        for (int i = 0; i < 16; ++i) sum[i] += attn_decode(code[i]);
        o[nb] = sum;
    }
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) st.o[nb] = o[nb];
}

// Scores of 32 keys from key0 on: -inf where the lane's row does not see the key.  Register i is key 8 (i / 4) + 4 hh + i % 4.
template <bool kBf16, int D>
__device__ __forceinline__ void attn_mask(const AttnRow<kBf16, D>& st, f32x16& s, int key0, uint32_t exists, int sinks, int hh) {
    const int from = st.lo - key0 - 4 * hh, to = st.hi - key0 - 4 * hh;
    if (key0 < sinks) {
        const int first = min(sinks - key0 - 4 * hh, to);
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            const int x = 8 * (i >> 2) + (i & 3);
            s[i] = (x >= from && x < to) || x < first ? s[i] : -INFINITY;
        }
    } else {
        const uint32_t span = (uint32_t)max(to - from, 0);
#pragma unroll
        for (int i = 0; i < 16; ++i) s[i] = (uint32_t)(8 * (i >> 2) + (i & 3) - from) < span ? s[i] : -INFINITY;
    }
    if ((exists & 3u) != 3u) {
#pragma unroll
        for (int i = 0; i < 16; ++i) s[i] = (exists >> (i >> 3)) & 1u ? s[i] : -INFINITY;
    }
}

// Bit i: the lane's row sees the key of register i.
template <bool kBf16, int D> __device__ __forceinline__ uint32_t attn_seen(const AttnRow<kBf16, D>& st, int key0, uint32_t exists, int sinks, int hh) {
    uint32_t seen = 0;
#pragma unroll 1
    for (int i = 0; i < 16; ++i) {
        const int key = key0 + 4 * hh + 8 * (i >> 2) + (i & 3);
        seen |= (key < st.hi && (key >= st.lo || key < sinks) && ((exists >> (i >> 3)) & 1u) ? 1u : 0u) << i;
    }
    return seen;
}

// 32 keys from key0 on for one wave.  full: every row sees all of them.  exists: bit g = keys 16g..16g+15 exist.  check: values may be not
// finite at keys that some row does not see (a product with a p of zero would be NaN).
template <bool kBf16, int D>
__device__ __forceinline__ void attn_block(const CacheAttnArgs& a, AttnRow<kBf16, D>& st, uint32_t k, uint32_t v, int key0, uint32_t exists,
                                           bool full, bool check, int hh) {
    constexpr int NB = D / 32, kRowB = AttnTile<kBf16, D>::kRowB;
    f32x16 s = attn_scores<kBf16, D>(st, k);
    if (!full) attn_mask<kBf16, D>(st, s, key0, exists, a.sinks, hh);
    float mx = s[0];
#pragma unroll
    for (int i = 1; i < 16; ++i) mx = fmaxf(mx, s[i]);
    mx *= a.scale_log2;
    if (__any(mx > st.ref + kAttnSlack)) attn_move_ref<kBf16, D>(st, mx);
    float sum = 0.0f;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
        s[i] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[i], a.scale_log2, st.sub));
        sum += s[i];
    }
    st.l += sum;
    if constexpr (kBf16) {
        bf16x8 p[2];   // operand of keys 16 kk ...: the lane half's are 16 kk + 8 (e / 4) + 4 hh + e % 4
#pragma unroll
        for (int kk = 0; kk < 2; ++kk)
#pragma unroll
            for (int e = 0; e < 8; ++e) p[kk][e] = (__bf16)s[8 * kk + e];
        if (!check || attn_finite<D>(v)) {
#pragma unroll
            for (int kk = 0; kk < 2; ++kk)
#pragma unroll
                for (int nb = 0; nb < NB; ++nb) {
                    st.o[nb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(attn_v<D>(v, kk, nb), p[kk], st.o[nb], 0, 0, 0);
                    if (nb & 1) __builtin_amdgcn_sched_barrier(0);   // or every operand is read at once, into registers that are not there
                }
        } else {
            attn_careful<D>(st, v, p, attn_seen<kBf16, D>(st, key0, exists, a.sinks, hh));
        }
    } else {
        // step i takes keys 8 (i / 4) + i % 4 of either lane half: register i is the operand
        auto operand = [&](int i, int nb) __attribute__((always_inline)) {
            return *(lds_f32_ptr)(uintptr_t)((v ^ (uint32_t)(nb << 7)) + (8 * (i >> 2) + (i & 3)) * kRowB);
        };
        bool plain = true;
        if (check) {
            f32x16 z;
#pragma unroll
            for (int i = 0; i < 16; ++i) z[i] = 0.0f;
#pragma unroll
            for (int i = 0; i < 16; ++i)
#pragma unroll
                for (int nb = 0; nb < NB; ++nb) {
                    z = __builtin_amdgcn_mfma_f32_32x32x2f32(operand(i, nb), 0.0f, z, 0, 0, 0);
                    if (nb == NB - 1 && i % 2) __builtin_amdgcn_sched_barrier(0);
                }
            float t = 0.0f;
#pragma unroll
            for (int i = 0; i < 16; ++i) t += z[i];
            plain = !__any(t != 0.0f);
        }
        if (plain) {
            float x[NB];
#pragma unroll
            for (int nb = 0; nb < NB; ++nb) x[nb] = operand(0, nb);
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                float next[NB];
#pragma unroll
                for (int nb = 0; nb < NB; ++nb) next[nb] = i + 1 < 16 ? operand(i + 1 < 16 ? i + 1 : i, nb) : x[nb];
#pragma unroll
                for (int nb = 0; nb < NB; ++nb) {
                    st.o[nb] = __builtin_amdgcn_mfma_f32_32x32x2f32(x[nb], s[i], st.o[nb], 0, 0, 0);
                    x[nb] = next[nb];
                }
                __builtin_amdgcn_sched_barrier(0);
            }
        } else {
            const uint32_t seen = attn_seen<kBf16, D>(st, key0, exists, a.sinks, hh);
            f32x16 o[NB];   // in memory, as above
#pragma unroll
            for (int nb = 0; nb < NB; ++nb) o[nb] = st.o[nb];
#pragma unroll 1
            for (int nb = 0; nb < NB; ++nb) {
                f32x16 sum = o[nb], code;
#pragma unroll
                for (int i = 0; i < 16; ++i) code[i] = 0.0f;
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    const float x = operand(i, nb), y = attn_code(x);
                    sum = __builtin_amdgcn_mfma_f32_32x32x2f32(y == 0.0f ? x : 0.0f, s[i], sum, 0, 0, 0);
                    code = __builtin_amdgcn_mfma_f32_32x32x2f32(y, attn_times(s[i], (seen >> i) & 1u), code, 0, 0, 0);
                }
#pragma unroll
                for (int i = 0; i < 16; ++i) sum[i] += attn_decode(code[i]);
                o[nb] = sum;
            }
#pragma unroll
            for (int nb = 0; nb < NB; ++nb) st.o[nb] = o[nb];
        }
    }
}

// A tile of 64 keys that every row of a wave sees, bf16, with the order of issue pinned: an MFMA holds the matrix pipe for 32 cycles, in
// whose shadow vector instructions issue (4 cycles each, 8 an exponential), so each segment below is one MFMA and what belongs
// under it.  Operand reads are issued kAhead MFMAs before their use.  The first scores' maximum and exponentials ride on the second
// block's products; the exponentials assume that the reference stays, and are formed again in the rare other case.  The other
// exponentials ride on the second product, 16 keys behind it.  (The same division of a step as the tile-sparse kernel's, attn_step.h; here
// V lies token by token, so its operand takes two transposing reads.)
template <int D> struct AttnStep {
    static constexpr int G = D / 16, NB = D / 32, kAhead = 6, kRowB = D * 2, NF = 2 * G + 4 * NB;
    static constexpr int kPieces = 4, kSeg = G / kPieces;   // block 0 comes in pieces, between which the caller asks for the next tile
    bf16x8 fr[NF], p[4];
    f32x16 s[2];
    float sum;
    uint32_t k, v;

    template <int F> __device__ __forceinline__ void read() {
        if constexpr (F < 2 * G) {
            fr[F] = *(lds_bf16x8_p)(uintptr_t)((k ^ (uint32_t)((F % G) << 5)) + (uint32_t)((F / G) * 32 * kRowB));
        } else if constexpr (F < NF) {
            constexpr int kk = (F - 2 * G) / NB, nb = (F - 2 * G) % NB;
            fr[F] = attn_v<D>(v, kk, nb);
        }
    }
    template <int F, int E> __device__ __forceinline__ void read_to() {
        if constexpr (F < E) { read<F>(); read_to<F + 1, E>(); }
    }
    __device__ __forceinline__ void begin(uint32_t k_at, uint32_t v_at) {
        k = k_at;
        v = v_at;
        read_to<0, kAhead>();
        __builtin_amdgcn_sched_barrier(0);
    }
    template <int F, int E> __device__ __forceinline__ void first(const AttnRow<true, D>& st) {
        if constexpr (F < E) {
            read<F + kAhead>();
            f32x16 z;
#pragma unroll
            for (int i = 0; i < 16; ++i) z[i] = 0.0f;
            s[0] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fr[F], st.qb[F], F == 0 ? z : s[0], 0, 0, 0);
            __builtin_amdgcn_sched_barrier(0);
            first<F + 1, E>(st);
        }
    }
    template <int P> __device__ __forceinline__ void piece(const AttnRow<true, D>& st) { first<P * kSeg, (P + 1) * kSeg>(st); }

    // exponentials of registers e, e + 1 of key step kk
    __device__ __forceinline__ void exp_pair(int kk, int e, float c, float sub, float& sum) {
        typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;
        const float p0 = __builtin_amdgcn_exp2f(__builtin_fmaf(s[kk >> 1][8 * (kk & 1) + e], c, sub));
        const float p1 = __builtin_amdgcn_exp2f(__builtin_fmaf(s[kk >> 1][8 * (kk & 1) + e + 1], c, sub));
        const bf16x2 pr = {(__bf16)p0, (__bf16)p1};
        sum += p0;
        sum += p1;
        // d = 64: here, under an MFMA; left to itself the compiler adds everything behind the last one.  d = 128: left to itself, its
        // shadows are full already (4680 rows x 12 heads, 34,320 keys, here / behind: 575 / 598 us at d = 64, 960 / 941 at 128).
        if constexpr (D == 64) asm volatile("" : "+v"(sum));
        p[kk][e] = pr[0];
        p[kk][e + 1] = pr[1];
    }
    static constexpr int kMaxSeg = G >= 8 ? 2 : 1, kExpSeg = G - 2 - kMaxSeg;   // block 0's last product needs two more to retire
    static_assert(kExpSeg >= 1 && 8 % kExpSeg == 0 && (8 / kExpSeg) % 2 == 0, "exponentials come in pairs");
    template <int F> __device__ __forceinline__ void second(const AttnRow<true, D>& st, float c, float& mx, float& sum) {
        if constexpr (F < 2 * G) {
            read<F + kAhead>();
            f32x16 z;
#pragma unroll
            for (int i = 0; i < 16; ++i) z[i] = 0.0f;
            s[1] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fr[F], st.qb[F - G], F == G ? z : s[1], 0, 0, 0);
            constexpr int i = F - G - 2;
            if constexpr (i >= 0 && i < kMaxSeg) {
#pragma unroll
                for (int e = i * (16 / kMaxSeg); e < (i + 1) * (16 / kMaxSeg); ++e) mx = fmaxf(mx, s[0][e]);
            }
            if constexpr (i >= kMaxSeg) {
#pragma unroll
                for (int e = (i - kMaxSeg) * (8 / kExpSeg); e < (i - kMaxSeg + 1) * (8 / kExpSeg); e += 2) exp_pair(0, e, c, st.sub, sum);
            }
            __builtin_amdgcn_sched_barrier(0);
            second<F + 1>(st, c, mx, sum);
        }
    }
    template <int I> __device__ __forceinline__ void third(AttnRow<true, D>& st, float c, float& sum) {
        if constexpr (I < 4 * NB) {
            constexpr int kk = I / NB, nb = I % NB;
            read<2 * G + I + kAhead>();
            st.o[nb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fr[2 * G + I], p[kk], st.o[nb], 0, 0, 0);
            if constexpr (kk < 3) {
#pragma unroll
                for (int e = nb * (8 / NB); e < (nb + 1) * (8 / NB); e += 2) exp_pair(kk + 1, e, c, st.sub, sum);
            }
            __builtin_amdgcn_sched_barrier(0);
            third<I + 1>(st, c, sum);
        }
    }
    // Scores of block 1.  false: some row's maximum has outgrown its reference, and nothing has been added to st.
    __device__ __forceinline__ bool scores(const AttnRow<true, D>& st, float c) {
        float mx = -INFINITY;
        sum = 0.0f;
        second<G>(st, c, mx, sum);
#pragma unroll
        for (int i = 0; i < 16; ++i) mx = fmaxf(mx, s[1][i]);
        return !__any(mx * c > st.ref + kAttnSlack);
    }
    __device__ __forceinline__ void values(AttnRow<true, D>& st, float c) {
        __builtin_amdgcn_s_setprio(1);   // a wave in its second product goes first: the SIMD's other one would delay these MFMAs
        __builtin_amdgcn_sched_barrier(0);
        third<0>(st, c, sum);
        __builtin_amdgcn_s_setprio(0);
        st.l += sum;
    }
};

template <bool kBf16, int D> struct AttnShape {
    typedef AttnTile<kBf16, D> T;
    static constexpr int kKeyTile = kBf16 ? 64 : 32;          // keys of a tile: one segment of loads a wave
    static constexpr int kSlot = 2 * kKeyTile * T::kRowB;     // K tile, V tile
    static constexpr int kOutRowB = T::kRowB + 16;            // a row of the results in LDS
    static constexpr int kOutB = kAttnRows * (kOutRowB + 4 + 8);   // and its lse, and where it goes
    static constexpr int kLds = 2 * kSlot > kOutB ? 2 * kSlot : kOutB;
};

// Pieces that unfinished sums can come in, at most (see the sharing kernel).
__device__ __forceinline__ int64_t rows_pieces(const CacheAttnArgs& a) { return 2 * (int64_t)a.workers + a.items * a.c.kv_heads; }

// Tiles t_beg .. t_end - 1 of those that rows r0 .. r_end - 1 of a sequence see, for one key head.  part: where the unfinished sums go,
// or -1 if these are all the tiles.
template <bool kBf16, int D>
__device__ __forceinline__ void rows_piece(const CacheAttnArgs& a, char* smem, int seq, const SeqRows& sr, int r0, int r_end, int head,
                                           const AttnTiles& tiles, int t_beg, int t_end, int64_t part) {
    typedef AttnShape<kBf16, D> Sh;
    typedef AttnTile<kBf16, D> T;
    constexpr int kRowB = T::kRowB, kKeyTile = Sh::kKeyTile, NB = D / 32;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int l31 = lane & 31, hh = lane >> 5;
    const int n = min(sr.n, a.c.max_new), rows = n * a.group;

    // the wave's rows
    const int w0 = r0 + 32 * wave;
    const bool active = w0 < rows;
    const int r = min(w0 + l31, rows - 1);
    AttnRow<kBf16, D> st;
    const char* q = a.q + (int64_t)(sr.first + r / a.group) * a.sq_n + (int64_t)(head * a.group + r % a.group) * a.sq_h;
    {
        const Seen v = seen_by(a, sr, n, r);
        st.lo = v.lo;
        st.hi = v.hi;
        if constexpr (kBf16) {
#pragma unroll
            for (int t = 0; t < D / 16; ++t) st.qb[t] = *reinterpret_cast<const bf16x8*>(q + 32 * t + 16 * hh);
        } else {
#pragma unroll
            for (int u = 0; u < D / 8; ++u) {
                const f32x4v x = *reinterpret_cast<const f32x4v*>(q + 32 * u + 16 * hh);
#pragma unroll
                for (int e = 0; e < 4; ++e) st.qf[4 * u + e] = x[e];
            }
        }
    }
    const int wave_lo = __builtin_amdgcn_readlane(st.lo, 0), wave_hi = __builtin_amdgcn_readlane(st.hi, 31);       // some row sees
    const int wave_lo_max = __builtin_amdgcn_readlane(st.lo, 31), wave_hi_min = __builtin_amdgcn_readlane(st.hi, 0);   // every row sees

    // Loads: lane i of a load lands at byte 16 i of its KB, so the swizzle is applied to what it fetches.
    // A segment's loads move on by 1 KB in either memory (the immediate offset), what is left of their swizzles is a constant each.
    const int load_row = lane / T::kChunks, load_c = lane % T::kChunks;
    const uint32_t k_off0 = (uint32_t)(load_row * kRowB + ((load_c ^ T::k_swizzle(load_row)) << 4));
    const uint32_t v_off0 = (uint32_t)(load_row * kRowB + ((load_c ^ T::v_swizzle(load_row)) << 4));
    const uint32_t lds = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)smem;
    const int64_t head_b = (int64_t)head * kRowB << a.c.log_page;
    const int page_mask = (1 << a.c.log_page) - 1;
    const int32_t* table = a.c.table + seq * a.c.table_stride;

    // Pages of the next 64 tiles, one tile a lane: looked up together, so that no step waits for the table.
    constexpr int kGroups = kKeyTile / 16;     // 16 keys never lie in two pages
    int32_t page = 0;                          // of the wave's segment
    uint32_t there = 0;                        // which of the groups exist
    auto look_up = [&](int t) {
        const int mine = t + lane, tok = tiles.at(mine);
        there = 0;
#pragma unroll
        for (int g = 0; g < kGroups; ++g) {
            const int at = tok + 16 * g;
            const int id = mine < t_end && at < sr.len ? table[at >> a.c.log_page] : -1;
            const bool ok = id >= 0 && id < a.c.pages;
            there |= (ok ? 1u : 0u) << g;
            if (g == wave * T::kSegRows / 16) page = ok ? id : 0;
        }
    };
    // asks for the wave's segment of tile t, number `at` of the pages looked up
    auto load_tile = [&](int t, int at, int slot) __attribute__((always_inline)) {
        const int row = wave * T::kSegRows, id = __builtin_amdgcn_readlane(page, at);
        const int64_t from = id * a.c.page_b + head_b + ((tiles.at(t) + row) & page_mask) * kRowB;
        const uint32_t to = lds + slot * Sh::kSlot + row * kRowB;
        uint32_t k_off[T::kSegLoads], v_off[T::kSegLoads];
#pragma unroll
        for (int j = 0; j < T::kSegLoads; ++j) {
            k_off[j] = k_off0 ^ T::k_step(j);
            v_off[j] = v_off0 ^ T::v_step(j);
        }
        dma16_group_to_lds<T::kSegLoads>(to, a.c.k + from, k_off);
        dma16_group_to_lds<T::kSegLoads>(to + kKeyTile * kRowB, a.c.v + from, v_off);
    };

    // the lane's part of operand addresses
    const uint32_t k_at = (uint32_t)(l31 * kRowB + ((hh ^ T::k_swizzle(l31)) << 4));
    uint32_t v_at;
    if constexpr (kBf16) {
        // transposing read: lane i of 16 names channels 4 (i % 4) ..+3 of key i / 4 and gets channel i of the four keys
        const int key = 4 * hh + ((lane >> 2) & 3), c = 2 * ((lane >> 4) & 1) + ((lane & 3) >> 1);
        v_at = (uint32_t)(key * kRowB + ((c ^ T::v_swizzle(key)) << 4) + 8 * (lane & 1));
    } else {
        v_at = (uint32_t)(4 * hh * kRowB + 4 * l31 + (hh << 7));
    }

    // Twice at most.  Values that are not finite at keys that exist are taken to be seen by all rows, or by none; where one turns up in
    // the sums, the workgroup does all of it again and looks at every tile that some row does not see whole.  (To look at once
    // costs as much as half of such a tile's products.)  Behind the sequence's end and in holes anything may lie: there it looks.
    float* ml = reinterpret_cast<float*>(smem + kAttnRows * Sh::kOutRowB);   // [128], and a flag of each wave before
    float l = 0.0f;
    for (bool careful = false;;) {
#pragma unroll
    for (int nb = 0; nb < NB; ++nb)
#pragma unroll
        for (int i = 0; i < 16; ++i) st.o[nb][i] = 0.0f;
    st.ref = -INFINITY;
    st.sub = st.l = 0.0f;
    int slot = 0, at = 0;
    if (t_beg < t_end) {
        look_up(t_beg);
        load_tile(t_beg, 0, 0);
    }
    // of 32 or 64 keys from `key` on: does some row see some, does every row see all of them
    auto some = [&](int key, int n, uint32_t ex) { return active && key < wave_hi && (key + n > wave_lo || key < a.sinks) && ex != 0; };
    auto all = [&](int key, int n, uint32_t ex) {
        return active && key + n <= wave_hi_min && (key >= wave_lo_max || key + n <= a.sinks) && ex == (1u << n / 16) - 1;
    };
    int t = t_beg, key0 = 0;
    uint32_t exists = 0;
    bool more = false, asked = false, started = false;   // asked: for tile t + 1
    // Tile t has landed in its slot and everyone has read the other one; look-up of the next.
    auto arrive = [&]() __attribute__((always_inline)) {
        exists = (uint32_t)__builtin_amdgcn_readlane((int)there, at);
        key0 = tiles.at(t);
        more = t + 1 < t_end;
        if (++at == 64 && more) {
            look_up(t + 1);
            at = 0;
        }
        __builtin_amdgcn_s_waitcnt(0xc07f);   // lgkmcnt(0): the other slot has been read
        wait_vmcnt<0>();
        asm volatile("" ::: "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
    };
    while (t < t_end) {
        arrive();
        if constexpr (kBf16) {
            // Tiles that every row sees, in a loop without any other path through the sums: with a branch that rescales them, or the
            // other kind of tile, in it, the compiler copies them from registers to registers at every step (64 of 224 vector
            // instructions).  So a tile for which a reference has to move leaves the loop and is done again below, and the first one
            // is done there at once.
            bool left = true;
            while (started && all(key0, 64, exists)) {
                const uint32_t base = lds + slot * Sh::kSlot;
                AttnStep<D> step;
                step.begin(base + k_at, base + v_at + kKeyTile * kRowB);
                step.template piece<0>(st);
                if (more) load_tile(t + 1, at, slot ^ 1);
                step.template piece<1>(st);
                step.template piece<2>(st);
                step.template piece<3>(st);
                asked = true;
                if (!step.scores(st, a.scale_log2)) break;
                step.values(st, a.scale_log2);
                asked = false;
                slot ^= 1;
                left = ++t < t_end;
                if (!left) break;
                arrive();
            }
            if (!left) break;
        }
        const uint32_t base = lds + slot * Sh::kSlot;
        if (more && !asked) load_tile(t + 1, at, slot ^ 1);
        asked = false;
        started = true;
#pragma unroll 1
        for (int c = 0; c < kKeyTile / 32; ++c) {
            const int key = key0 + 32 * c;
            const uint32_t ex = (exists >> (2 * c)) & 3u;
            if (some(key, 32, ex)) {
                const bool full = all(key, 32, ex);
                attn_block<kBf16, D>(a, st, base + k_at + c * 32 * kRowB, base + v_at + (kKeyTile + c * 32) * kRowB, key, ex, full,
                                     !full && (careful || ex != 3u || key + 32 > sr.len), hh);
            }
        }
        ++t;
        slot ^= 1;
    }

    l = sum_with_other_half(st.l);
    if (careful) break;
    float odd = 0.0f * l;
#pragma unroll
    for (int nb = 0; nb < NB; ++nb)
#pragma unroll
        for (int i = 0; i < 16; ++i) odd = __builtin_fmaf(st.o[nb][i], 0.0f, odd);
    __syncthreads();
    if (lane == 0) ml[wave] = 0.0f;
    if (odd != 0.0f) ml[wave] = 1.0f;   // NaN
    __syncthreads();
    if (ml[0] + ml[1] + ml[2] + ml[3] == 0.0f) break;
    careful = true;
    __syncthreads();
    }

    // Results.  A lane holds channels 32 nb + 8 j + 4 hh + 0..3 of its row.
    __syncthreads();
    char* orow = smem + (wave * 32 + l31) * Sh::kOutRowB;
    if (part >= 0) {   // [part][row][D] sums, then [part][row] reference and l
        if (w0 + l31 < r_end) {
            const int64_t row = part * a.part_rows + 32 * wave + l31;
            float* po = a.part + row * D;
#pragma unroll
            for (int nb = 0; nb < NB; ++nb)
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    *reinterpret_cast<f32x4v*>(po + 32 * nb + 8 * j + 4 * hh) = f32x4v{st.o[nb][4 * j], st.o[nb][4 * j + 1], st.o[nb][4 * j + 2], st.o[nb][4 * j + 3]};
            if (hh == 0) *reinterpret_cast<float2*>(a.part + rows_pieces(a) * a.part_rows * D + row * 2) = float2{st.ref, l};
        }
        return;
    }
    const float inv = attn_inverse(a, seq, sr, r, l);
#pragma unroll
    for (int nb = 0; nb < NB; ++nb)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int ch = 32 * nb + 8 * j + 4 * hh;
            if constexpr (kBf16) {
                bf16x4 x;
#pragma unroll
                for (int e = 0; e < 4; ++e) x[e] = (__bf16)(st.o[nb][4 * j + e] * inv);
                *reinterpret_cast<bf16x4*>(orow + ch * 2) = x;
            } else {
                *reinterpret_cast<f32x4v*>(orow + ch * 4) = f32x4v{st.o[nb][4 * j] * inv, st.o[nb][4 * j + 1] * inv, st.o[nb][4 * j + 2] * inv, st.o[nb][4 * j + 3] * inv};
            }
        }
    char** to = reinterpret_cast<char**>(ml + kAttnRows);
    if (hh == 0) ml[wave * 32 + l31] = attn_lse(st.ref, l);
    if (tid < r_end - r0) {
        const int at_row = r0 + tid;
        to[tid] = a.out + (int64_t)(sr.first + at_row / a.group) * a.so_n + (int64_t)(head * a.group + at_row % a.group) * a.so_h;
    }
    __syncthreads();
    // Past the caches, and rows' places found once each: prompts as above 328 us instead of 336.
    int me = tid;
    asm volatile("" : "+v"(me));   // or the sharing kernel keeps what follows from it in registers, from piece to piece
#pragma unroll
    for (int j = 0; j < kAttnRows * T::kChunks / 256; ++j) {
        const int rr = (j * 256 + me) / T::kChunks, c = me % T::kChunks;
        if (rr < r_end - r0) store_through(to[rr] + 16 * c, *reinterpret_cast<const uint4*>(smem + rr * Sh::kOutRowB + 16 * c));
    }
    if (a.lse && tid < r_end - r0) {
        const int at_row = r0 + tid;
        a.lse[(int64_t)(head * a.group + at_row % a.group) * a.c.rows + sr.first + at_row / a.group] = ml[tid];
    }
}

// A workgroup for each (block of rows, key head).  Heads next to each other: workgroups are dealt to the 8 dies in turn, so those of
// a head meet in few L2 caches.
template <bool kBf16, int D> __global__ __launch_bounds__(256, 2) void cache_attn_rows_kernel(CacheAttnArgs a) {
    extern __shared__ __align__(1024) char smem[];
    RowBlock rb;
    if (!block_of(a.c, a.group, kAttnRows, a.per_seq, blockIdx.x / a.c.kv_heads, rb)) return;
    const SeqRows sr = rb.rows;
    const int rows = min(sr.n, a.c.max_new) * a.group;
    const int r0 = (rb.blocks - 1 - rb.block) * kAttnRows;   // the last rows of a causal sequence see the most
    const int r_end = min(rows, r0 + kAttnRows);
    const AttnTiles tiles = tiles_seen(a, sr, min(sr.n, a.c.max_new), r0, r_end - 1, AttnShape<kBf16, D>::kKeyTile);
    rows_piece<kBf16, D>(a, smem, rb.seq, sr, r0, r_end, blockIdx.x % a.c.kv_heads, tiles, 0, tiles.count, -1);
}

// Where there are few blocks, a workgroup for each leaves compute units idle, so their tiles are dealt out to as many workgroups as fit the
// card at once, all with the same number of tiles, `level`.  Of every block's list the first whole multiples of `level` go to workgroups of
// their own: piece k of every block walks the same tiles of its head at the same time, out of the dies' L2.  (Pieces that
// merely lie one behind the other, each beginning where the last one ended, do not: 12 heads of 37 blocks, 444 on 512 places, 1.04 ms instead of
// 0.90 with a workgroup for each.)  What is left of the lists is laid end to end and shared by the other workgroups, where every piece counts
// for kPiece tiles more: what its set-up and its sums' way to the workspace take (fp32, 1057 rows x 12 heads in 28 blocks on 2000 keys, with 0 / 2 / 5:
// 142 / 117 / 116 us, 449 rows 64 / 64 / 71; bf16, 2560 rows x 12 heads on 34,000 keys with 0 / 1 / 3: 531 / 491 / 492, 3840 rows 729 / 734 /
// 752).  Every workgroup counts the blocks' tiles itself.
template <int kTile> __device__ __forceinline__ int rows_tiles_of(const CacheAttnArgs& a, int item) {
    if (item >= a.items) return 0;
    const SeqRows sr = seq_rows(a.c, item / a.per_seq);
    const int n = min(sr.n, a.c.max_new), rows = n * a.group, r0 = item % a.per_seq * kAttnRows;
    return r0 >= rows ? 0 : max(1, tiles_seen(a, sr, n, r0, min(rows, r0 + kAttnRows) - 1, kTile).count);
}
constexpr int kRowsShareTiles = 4;   // least level
// Number of a piece of unfinished sums: whole multiples by workgroup, the others (block and workgroup both only grow from one to the next)
// by their sum.
__device__ __forceinline__ int64_t rows_piece_id(const CacheAttnArgs& a, int parts, int item, int q, int head) {
    return (int64_t)(q < 0 ? item : parts + item + q) * a.c.kv_heads + head;
}
template <int D> __device__ __forceinline__ int4* rows_cuts(const CacheAttnArgs& a) {
    return reinterpret_cast<int4*>(a.part + rows_pieces(a) * a.part_rows * (D + 2));
}

template <bool kBf16, int D> __global__ __launch_bounds__(256, 2) void cache_attn_rows_share_kernel(CacheAttnArgs a) {
    constexpr int kTile = AttnShape<kBf16, D>::kKeyTile, kPiece = kBf16 ? 1 : 2;
    extern __shared__ __align__(1024) char smem[];
    auto rest_units = [](int tiles) { return tiles ? tiles + kPiece : 0; };
    const int lane = threadIdx.x & 63, head = blockIdx.x % a.c.kv_heads, mine = blockIdx.x / a.c.kv_heads, parts = a.workers / a.c.kv_heads;
    auto sum = [&](int x) { return __builtin_amdgcn_readlane(lanes_up_to(x), 63); };
    int counts[kRowsShareItems / 64];
    int total = 0;
#pragma unroll
    for (int k = 0; k < kRowsShareItems / 64; ++k) {
        counts[k] = 64 * k < a.items ? rows_tiles_of<kTile>(a, 64 * k + lane) : 0;
        total += sum(counts[k]);
    }
    int level = max(kRowsShareTiles, (total + parts - 1) / parts), fulls, units;
    for (;; level += (level + 15) / 16) {
        int f = 0, u = 0;
#pragma unroll
        for (int k = 0; k < kRowsShareItems / 64; ++k) {
            f += counts[k] / level;
            u += rest_units(counts[k] % level);
        }
        fulls = sum(f);
        units = sum(u);
        if (fulls + (units + level + kPiece - 1) / (level + kPiece) <= parts) break;
    }
    const TileShare rests(units, parts - fulls, 1);
    const bool full = mine < fulls;
    const int q = full ? -1 : mine - fulls;
    if (!full && (units == 0 || q >= rests.parts)) return;
    // the block: of the whole multiples, number `mine`; of what is left, the one that unit `now` of it falls into
    int now = full ? 0 : rests.begin(q), item = 0, first_full = 0, first_unit = 0;
    const int end = full ? 1 : rests.begin(q + 1);
    bool found = false;
#pragma unroll
    for (int k = 0; k < kRowsShareItems / 64; ++k) {
        const int f = counts[k] / level, u = rest_units(counts[k] % level), up_f = lanes_up_to(f), up_u = lanes_up_to(u);
        const int all_f = __builtin_amdgcn_readlane(up_f, 63), all_u = __builtin_amdgcn_readlane(up_u, 63);
        if (found) continue;
        found = full ? mine < first_full + all_f : now < first_unit + all_u;
        if (found) {
            const int at = __popcll(__ballot(full ? first_full + up_f <= mine : first_unit + up_u <= now));
            item = 64 * k + at;
            first_full += __builtin_amdgcn_readlane(up_f, at) - __builtin_amdgcn_readlane(f, at);
            first_unit += __builtin_amdgcn_readlane(up_u, at) - __builtin_amdgcn_readlane(u, at);
        } else {
            first_full += all_f;
            first_unit += all_u;
        }
    }
    for (bool again = false; now < end && item < a.items; ++item) {
        const int seq = item / a.per_seq;
        const SeqRows sr = seq_rows(a.c, seq);
        const int n = min(sr.n, a.c.max_new), rows = n * a.group, r0 = item % a.per_seq * kAttnRows;
        if (r0 >= rows) continue;
        const int r_end = min(rows, r0 + kAttnRows);
        const AttnTiles tiles = tiles_seen(a, sr, n, r0, r_end - 1, kTile);
        const int count = max(1, tiles.count), f = count / level, rest = count - f * level, next_unit = first_unit + rest_units(rest);
        // tiles of this piece
        const int t_beg = full ? (mine - first_full) * level : f * level + max(0, now - first_unit - kPiece);
        const int t_end = full ? t_beg + level : f * level + max(0, min(end, next_unit) - first_unit - kPiece);
        if (t_end > t_beg) {
            const bool whole = t_beg == 0 && t_end == count;
            if (t_beg == 0 && threadIdx.x == 0) {   // whole multiples: how many, from which workgroup on; then the others
                const int q0 = rest ? rests.owner(first_unit + kPiece) : 0, q1 = rest ? rests.owner(next_unit - 1) : -1;
                rows_cuts<D>(a)[item * a.c.kv_heads + head] = int4{whole ? 0 : f, first_full, whole ? 0 : q1 - q0 + 1, q0};
            }
            if (again) __syncthreads();   // the last piece's results have left the slots
            rows_piece<kBf16, D>(a, smem, seq, sr, r0, r_end, head, tiles, t_beg, min(t_end, tiles.count), whole ? -1 : rows_piece_id(a, parts, full ? mine : item, q, head));
            again = true;
        }
        now = full ? end : max(now, min(end, next_unit));
        first_unit = next_unit;
        first_full += f;
    }
}

// Puts a cut block's unfinished sums together, four rows a workgroup: its waves take every fourth piece.
template <bool kBf16, int D> __global__ __launch_bounds__(256) void cache_attn_rows_join_kernel(CacheAttnArgs a) {
    constexpr int V = D / 64;
    __shared__ float sums[4][4][D + 2];
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, head = blockIdx.x % a.c.kv_heads, item = blockIdx.x / a.c.kv_heads;
    const SeqRows sr = seq_rows(a.c, item / a.per_seq);
    const int block_rows = min(min(sr.n, a.c.max_new) * a.group - item % a.per_seq * kAttnRows, kAttnRows), r0 = 4 * blockIdx.y, rows = min(4, block_rows - r0);
    if (rows <= 0) return;
    const int4 cut = rows_cuts<D>(a)[blockIdx.x];
    const int n = cut.x + cut.z, parts = a.workers / a.c.kv_heads;
    if (n == 0) return;   // one workgroup had it whole
    const float2* ml = reinterpret_cast<const float2*>(a.part + rows_pieces(a) * a.part_rows * D);
    auto part_row = [&](int j, int r) {
        const int64_t id = j < cut.x ? rows_piece_id(a, parts, cut.y + j, -1, head) : rows_piece_id(a, parts, item, cut.w + j - cut.x, head);
        return id * a.part_rows + r0 + min(r, rows - 1);
    };
    float ref[4], l[4], o[4][V];
#pragma unroll
    for (int r = 0; r < 4; ++r) {
        ref[r] = -INFINITY;
        l[r] = 0.0f;
#pragma unroll
        for (int c = 0; c < V; ++c) o[r][c] = 0.0f;
    }
    for (int j = lane; j < n; j += 64)
#pragma unroll
        for (int r = 0; r < 4; ++r) ref[r] = fmaxf(ref[r], ml[part_row(j, r)].x);
#pragma unroll
    for (int r = 0; r < 4; ++r)
#pragma unroll
        for (int x = 32; x >= 1; x >>= 1) ref[r] = fmaxf(ref[r], __shfl_xor(ref[r], x));
    for (int j = wave; j < n; j += 4) {
        float2 m[4];
        float x[4][V];
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const int64_t at = part_row(j, r);
            m[r] = ml[at];
#pragma unroll
            for (int c = 0; c < V; ++c) x[r][c] = a.part[at * D + V * lane + c];
        }
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const float f = m[r].x == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(m[r].x - ref[r]);   // -inf: the sums are 0 or NaN
            l[r] += f * m[r].y;
#pragma unroll
            for (int c = 0; c < V; ++c) o[r][c] += f * x[r][c];
        }
    }
#pragma unroll
    for (int r = 0; r < 4; ++r) {
#pragma unroll
        for (int c = 0; c < V; ++c) sums[wave][r][V * lane + c] = o[r][c];
        if (lane == 0) sums[wave][r][D] = l[r];
    }
    __syncthreads();
    if (wave >= rows) return;   // one wave for each row from here on
    float lsum = 0.0f, y[V];
#pragma unroll
    for (int c = 0; c < V; ++c) y[c] = 0.0f;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
        lsum += sums[w][wave][D];
#pragma unroll
        for (int c = 0; c < V; ++c) y[c] += sums[w][wave][V * lane + c];
    }
    const int row = item % a.per_seq * kAttnRows + r0 + wave, qh = head * a.group + row % a.group;
    const float inv = attn_inverse(a, item / a.per_seq, sr, row, lsum);
    const int64_t token = sr.first + row / a.group;
    char* dst = a.out + token * a.so_n + (int64_t)qh * a.so_h;
#pragma unroll
    for (int c = 0; c < V; ++c) {
        if constexpr (kBf16) reinterpret_cast<__bf16*>(dst)[V * lane + c] = (__bf16)(y[c] * inv);
        else reinterpret_cast<float*>(dst)[V * lane + c] = y[c] * inv;
    }
    const float top = wave == 0 ? ref[0] : wave == 1 ? ref[1] : wave == 2 ? ref[2] : ref[3];
    if (a.lse && lane == 0) a.lse[(int64_t)qh * a.c.rows + token] = attn_lse(top, lsum);
}

template <bool kBf16, int D> static veda_status launch_rows(const CacheAttnArgs& a, hipStream_t s) {
    typedef AttnShape<kBf16, D> Sh;
    auto kern = a.workers ? cache_attn_rows_share_kernel<kBf16, D> : cache_attn_rows_kernel<kBf16, D>;
    if (Sh::kLds > 64 * 1024) VEDA_HIP_TRY(hipFuncSetAttribute((const void*)kern, hipFuncAttributeMaxDynamicSharedMemorySize, Sh::kLds));
    hipLaunchKernelGGL(kern, dim3((unsigned)(a.workers ? a.workers : a.items * a.c.kv_heads)), dim3(256), Sh::kLds, s, a);
    const veda_status st = launch_status("veda_cache_attn_fwd");
    if (st != VEDA_OK || !a.workers) return st;
    hipLaunchKernelGGL((cache_attn_rows_join_kernel<kBf16, D>), dim3((unsigned)(a.items * a.c.kv_heads), (unsigned)((a.part_rows + 3) / 4)), dim3(256), 0, s, a);
    return launch_status("veda_cache_attn_fwd");
}

// Two workgroups fit a compute unit, by LDS and registers alike.  bf16 shares among so many: one's products run while the other waits.  fp32
// products leave no such gaps, and half the workgroups have half the unfinished sums to write and join (12 heads on 4 key heads, d = 128, us
// with 512 / 256: 449 rows on 2000 keys 72 / 63, on 8300 194 / 195, 129 rows on 3100 56 / 45; bf16, 1280 rows on 34,000 keys 285 / 368).
int attn_rows_places() { return 512; }
int attn_rows_workers(bool bf16) { return bf16 ? 512 : 256; }

veda_status launch_cache_attn_rows(const CacheAttnArgs& a, bool bf16, int d, hipStream_t s) {
    if (bf16) return d == 128 ? launch_rows<true, 128>(a, s) : launch_rows<true, 64>(a, s);
    return d == 128 ? launch_rows<false, 128>(a, s) : launch_rows<false, 64>(a, s);
}

}  // namespace veda
