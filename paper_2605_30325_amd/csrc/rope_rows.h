// Rotary positions on rows of channels: the handle, the angles of a block of tokens, and the pass over its rows, shared by
// the calls that rotate (rope.hip, cache.hip).  Not part of the public ABI.
//
// y0 = A (x0 cos - x1 sin), y1 = A (x0 sin + x1 cos) for every pair of channels: 2 bytes moved for each flop or so, so memory
// bounds it, and everything here serves 16-byte accesses and few instructions between them.  The angle of a pair is the same
// for all heads of a token: a workgroup takes a block of tokens with as many heads as there are, puts A cos and A sin of the
// block into LDS once and streams the heads' rows past them.  32,760 tokens x 40 heads of 128 channels, bf16, three axes: 136 us = 4.9 TB/s
// (a large copy: 5.0); a chunk of 4680 x 36 rows into the cache 18 us = 4.8 TB/s.
#pragma once

#include "store.h"
#include "veda_internal.h"

struct veda_rope {
    veda_rope_config cfg;
    int32_t rot = 0;               // channels that rotate
    double amplitude = 1.0;
    std::vector<double> freq;      // radians per position
    double* d_turns = nullptr;     // device [rot / 2]: turns per position
    int device = -1;
};

namespace veda {

#if defined(__HIPCC__)

struct RopeArgs {
    const double* turns;   // null: rows are copied
    int32_t half;          // pairs: rot / 2
    int32_t end0, end1;    // pairs of axis 0, and of axes 0 and 1
    int32_t axes, halves;
    float amplitude;
    float sign;            // -1: the transposed matrix
    int32_t through;       // stores go past the caches
};

inline RopeArgs rope_args(const veda_rope* r, int transpose) {
    RopeArgs a{nullptr, 0, 0, 0, 1, 0, 1.0f, 1.0f, 0};
    if (!r) return a;
    a.turns = r->d_turns;
    a.half = r->rot / 2;
    a.axes = r->cfg.axes;
    a.end0 = r->cfg.axis_dim[0] / 2;
    a.end1 = a.end0 + (a.axes > 1 ? r->cfg.axis_dim[1] / 2 : 0);
    a.halves = r->cfg.pairs == VEDA_ROPE_HALVES;
    a.amplitude = (float)r->amplitude;
    a.sign = transpose ? -1.0f : 1.0f;
    return a;
}

// Whether 16-byte chunks never straddle what the rotation tells apart: the two halves of the pairs, or the rotated and the
// copied channels.
inline bool rope_in_chunks(const RopeArgs& a, int chunk) { return (a.halves ? a.half : 2 * a.half) % chunk == 0; }

// Whether what neighbouring threads store at a time, a row or the pieces that its units begin and end in, is whole lines of 128 bytes.  Such stores
// are better not kept in the caches (32,760 x 40 rows of 128 bf16 136 us instead of 139, fp32 127 instead of 137), others meet
// there: 32,760 x 80 rows of 64 of which 32 rotate, in halves, 150 us instead of 204 past them, 16,200 x 40 appended rows of 64 31 instead of 36.
inline bool rope_whole_lines(const RopeArgs& a, int head_dim, int es) {
    return a.halves ? a.half * es % 128 == 0 && (head_dim - 2 * a.half) * es % 128 == 0 : head_dim * es % 128 == 0;
}

// Units of a row: what one thread loads, turns and stores at a time.  In chunks: two chunks of pairs (halves) or one
// (interleaved), or one copied chunk.  Otherwise a pair of channels or one copied channel.
inline int rope_units(const RopeArgs& a, int head_dim, int chunk, bool in_chunks) {
    if (!in_chunks) return a.half + head_dim - 2 * a.half;
    return a.halves ? a.half / chunk + (head_dim - 2 * a.half) / chunk : head_dim / chunk;
}

constexpr int kRopeThreads = 256;

// A cos and A sin of tokens 0..n-1 of a block, [token][pair]; pos(t, axis) is a token's position.
// The product position * turns is formed in 64 bits and only its fraction kept: fp32 would be off by a radian's part at
// positions of 2^20 already.  What the fraction loses as fp32, up to 2^-26 of a turn, 1.6 half steps of a sine near 1, is put back to first order.
template <typename Pos> __device__ __forceinline__ void rope_angles(const RopeArgs& a, int n, Pos pos, float2* cs) {
    for (int i = threadIdx.x; i < n * a.half; i += kRopeThreads) {
        const int t = i / a.half, p = i % a.half;
        const double turns = (double)pos(t, p < a.end0 ? 0 : p < a.end1 ? 1 : 2) * a.turns[p];
        const double part = turns - rint(turns);
        float s, c;
        sincospif(2.0f * (float)part, &s, &c);
        const float rest = 6.2831853f * (float)(part - (double)(float)part);
        cs[i] = float2{a.amplitude * (c - s * rest), a.sign * a.amplitude * (s + c * rest)};
    }
}

template <typename E> struct RopeChunk;
template <> struct RopeChunk<uint16_t> {
    static constexpr int kN = 8;
    __device__ static void unpack(const uint4& u, float* f) { Chunk<uint16_t>::unpack(u, f); }
    __device__ static uint4 pack(const float* f) {
        typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8;
        bf16x8 v;
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = (__bf16)f[i];
        return __builtin_bit_cast(uint4, v);
    }
    __device__ static float load(const char* p) { return __uint_as_float((uint32_t)*reinterpret_cast<const uint16_t*>(p) << 16); }
    __device__ static void store(char* p, float x) { *reinterpret_cast<uint16_t*>(p) = __builtin_bit_cast(uint16_t, (__bf16)x); }
};
template <> struct RopeChunk<uint32_t> {
    static constexpr int kN = 4;
    __device__ static void unpack(const uint4& u, float* f) { Chunk<uint32_t>::unpack(u, f); }
    __device__ static uint4 pack(const float* f) {
        return uint4{__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3])};
    }
    __device__ static float load(const char* p) { return *reinterpret_cast<const float*>(p); }
    __device__ static void store(char* p, float x) { *reinterpret_cast<float*>(p) = x; }
};

struct RowMove {
    const char* src;
    char* dst;         // null: nothing to do
    int token;         // of the block
    bool turn;
};

// The order in which a workgroup goes through its rows: the heads of a token one after the other where they lie next to each other
// ([tokens][heads][channels]), else the tokens of a head.
struct RowOrder { int32_t heads_first; };
inline RowOrder row_order(bool heads_first) { return RowOrder{heads_first ? 1 : 0}; }
struct RowAt {
    bool heads_first;
    int log_tb, heads;
    uint32_t magic;    // 2^32 / heads, rounded up: exact quotients while row * heads < 2^32 (16 tokens, 256 heads)
    __device__ __forceinline__ RowAt(const RowOrder& o, int log_tb_, int heads_)
        : heads_first(o.heads_first && heads_ > 1), log_tb(log_tb_), heads(heads_), magic(0xffffffffu / (uint32_t)heads_ + 1u) {}
    __device__ __forceinline__ int rows(int tokens) const { return heads_first ? tokens * heads : heads << log_tb; }
    __device__ __forceinline__ void find(int r, int& t, int& h) const {
        if (heads_first) {
            t = (int)__umulhi((uint32_t)r, magic);
            h = r - t * heads;
        } else {
            t = r & ((1 << log_tb) - 1);
            h = r >> log_tb;
        }
    }
};

// Rows 0..n_rows-1 of a block: move(r) tells where row r lies and goes, its token in the block and whether it turns.
// A thread keeps one unit of the row and goes from row to row, kAhead of them at a time so that their loads are in flight
// together (two: four and eight cost more waves than they bring, 140 against 155 and 187 us for 32,760 x 40 rows of 128); a unit is loaded whole before any of it is stored, and no two units touch the same bytes (rows may be turned in place).
template <typename E, bool kChunks, typename Move>
__device__ __forceinline__ void rope_rows(const RopeArgs& a, int head_dim, int units, int n_rows, const float2* cs, Move move) {
    typedef RopeChunk<E> C;
    constexpr int kN = C::kN, kAhead = 2, es = sizeof(E);
    const int width = units < kRopeThreads ? units : kRopeThreads, step = kRopeThreads / width;
    const int r0 = threadIdx.x / width;
    if (r0 >= step) return;
    for (int u = threadIdx.x % width; u < units; u += width) {
        if constexpr (kChunks) {
            const int paired = a.halves ? a.half / kN : 0;           // units of two chunks
            const bool two = u < paired, turns = two || (!a.halves && u * kN < 2 * a.half);
            const int c0 = a.halves && !two ? u + paired : u, c1 = u + paired;
            const int pair0 = a.halves ? u * kN : u * (kN / 2);
            for (int r = r0; r < n_rows; r += kAhead * step) {
                uint4 x[kAhead], y[kAhead];
                RowMove m[kAhead];
#pragma unroll
                for (int j = 0; j < kAhead; ++j) {
                    m[j].dst = nullptr;
                    if (r + j * step < n_rows) m[j] = move(r + j * step);
                    if (!m[j].dst) continue;
                    x[j] = *reinterpret_cast<const uint4*>(m[j].src + c0 * 16);
                    if (two) y[j] = *reinterpret_cast<const uint4*>(m[j].src + c1 * 16);
                }
#pragma unroll
                for (int j = 0; j < kAhead; ++j) {
                    if (!m[j].dst) continue;
                    if (turns && m[j].turn) {
                        const float2* w = cs + m[j].token * a.half + pair0;
                        float f[kN];
                        C::unpack(x[j], f);
                        if (two) {
                            float g[kN];
                            C::unpack(y[j], g);
#pragma unroll
                            for (int e = 0; e < kN; ++e) {
                                const float2 z = w[e];
                                const float p = f[e] * z.x - g[e] * z.y;
                                g[e] = f[e] * z.y + g[e] * z.x;
                                f[e] = p;
                            }
                            y[j] = C::pack(g);
                        } else {
#pragma unroll
                            for (int e = 0; e < kN / 2; ++e) {
                                const float2 z = w[e];
                                const float p = f[2 * e] * z.x - f[2 * e + 1] * z.y;
                                f[2 * e + 1] = f[2 * e] * z.y + f[2 * e + 1] * z.x;
                                f[2 * e] = p;
                            }
                        }
                        x[j] = C::pack(f);
                    }
                    if (a.through) {
                        store_through(m[j].dst + c0 * 16, x[j]);
                        if (two) store_through(m[j].dst + c1 * 16, y[j]);
                    } else {
                        *reinterpret_cast<uint4*>(m[j].dst + c0 * 16) = x[j];
                        if (two) *reinterpret_cast<uint4*>(m[j].dst + c1 * 16) = y[j];
                    }
                }
            }
        } else {
            const bool pair = u < a.half;
            const int c0 = pair ? (a.halves ? u : 2 * u) : u + a.half, c1 = a.halves ? u + a.half : 2 * u + 1;
            for (int r = r0; r < n_rows; r += step) {
                const RowMove m = move(r);
                if (!m.dst) continue;
                const float x0 = C::load(m.src + c0 * es);
                if (!pair) {
                    C::store(m.dst + c0 * es, x0);
                    continue;
                }
                const float x1 = C::load(m.src + c1 * es);
                float2 z{1.0f, 0.0f};
                if (m.turn) z = cs[m.token * a.half + u];
                C::store(m.dst + c0 * es, m.turn ? x0 * z.x - x1 * z.y : x0);
                C::store(m.dst + c1 * es, m.turn ? x0 * z.y + x1 * z.x : x1);
            }
        }
    }
}

// Tokens of a block (a power of two) and heads of a workgroup: blocks of 16 tokens with up to 256 heads, and less of both until there
// are four workgroups to a compute unit or a workgroup has one token and four heads.
inline void rope_blocks(int64_t tokens, int64_t samples, int64_t heads, int* log_tb, int* hb) {
    *log_tb = 4;
    while (*log_tb > 0 && (tokens >> (*log_tb - 1)) <= 1) --*log_tb;
    int64_t h = heads < 256 ? heads : 256;
    auto blocks = [&] { return samples * ((tokens + (1 << *log_tb) - 1) >> *log_tb) * ((heads + h - 1) / h); };
    while (blocks() < 1024 && h > 4) h = (h + 1) / 2;
    while (blocks() < 1024 && *log_tb > 0) --*log_tb;
    *hb = (int)h;
}

#endif

}  // namespace veda
