// The paged cache held in 4 bits: checks, rounding and appending the newest rows, copies of pages.
#include "packed.h"
#include "rope_rows.h"

namespace veda {

veda_status check_packed(const veda_packed_cache* c) {
    if (!c || !c->k || !c->v || c->pages < 1 || c->kv_heads < 1 || c->page_stride < 0) return VEDA_ERR_INVALID_ARG;
    if (c->dtype != VEDA_F32 && c->dtype != VEDA_BF16) return VEDA_ERR_INVALID_ARG;
    if (c->head_dim != 64 && c->head_dim != 128) return VEDA_ERR_UNSUPPORTED;
    if (c->kv_heads > 1024) return VEDA_ERR_UNSUPPORTED;
    if (c->page_tokens < 16 || c->page_tokens > 256 || (c->page_tokens & (c->page_tokens - 1))) return VEDA_ERR_UNSUPPORTED;
    if (c->page_stride && c->page_stride < c->kv_heads * packed_head_bytes(c)) return VEDA_ERR_INVALID_ARG;
    if (c->page_stride % 16 || !aligned16(c->k) || !aligned16(c->v)) return VEDA_ERR_UNSUPPORTED;
    return VEDA_OK;
}

veda_cache packed_rows(const veda_packed_cache* c) {
    return veda_cache{c->pages, c->page_tokens, c->kv_heads, c->head_dim, c->dtype, 0, c->k, c->v};
}

CacheArgs packed_args(const veda_packed_cache* c, const veda_cache_batch* b) {
    const veda_cache rows = packed_rows(c);
    CacheArgs a = cache_args(&rows, b);
    a.page_b = c->page_stride ? c->page_stride : c->kv_heads * packed_head_bytes(c);
    return a;
}

struct PackedAppendArgs {
    CacheArgs c;
    RopeArgs rope;
    double amplitude;
    const char *q, *k, *v;
    char *q_out, *k_out, *v_out;
    int64_t sq_h, sq_n, so_h, so_n, sk_h, sk_n, sv_h, sv_n, sko_h, sko_n, svo_h, svo_n;   // bytes
    const int32_t* positions;   // null: the position in the sequence
    int64_t head_b;             // bytes of a head in a page
    int32_t q_heads, head_dim, units, log_tb, hb, q_groups, per_seq;
    RowOrder order;
};

// A cos and A sin of the block's tokens in 64 bits, for values that a code's border decides about.
template <typename Pos> __device__ __forceinline__ void packed_angles(const RopeArgs& a, double amplitude, int n, Pos pos, double2* cs) {
    for (int i = threadIdx.x; i < n * a.half; i += kRopeThreads) {
        const int t = i / a.half, p = i % a.half;
        const double turns = (double)pos(t, p < a.end0 ? 0 : p < a.end1 ? 1 : 2) * a.turns[p];
        double s, c;
        sincospi(2.0 * (turns - rint(turns)), &s, &c);
        cs[i] = double2{amplitude * c, amplitude * s};
    }
}

// x to fp32 by rounding to odd: what is inexact lies strictly between the same fp32 numbers of few bits, the codes' borders among them, as
// before, so that rounding it once more gives what rounding x gives.
__device__ __forceinline__ float packed_odd(double x) {
    const float f = (float)x;
    uint32_t u = __float_as_uint(f);
    if ((double)f != x) u = (u - (fabsf(f) > fabs(x) ? 1u : 0u)) | 1u;
    return __uint_as_float(u);
}

// Eight channels from p on.
__device__ __forceinline__ void packed_load(const uint16_t*, const char* p, float (&f)[8]) { Chunk<uint16_t>::unpack(*reinterpret_cast<const uint4*>(p), f); }
__device__ __forceinline__ void packed_load(const uint32_t*, const char* p, float (&f)[8]) {
    const uint4 x = reinterpret_cast<const uint4*>(p)[0], y = reinterpret_cast<const uint4*>(p)[1];
    const uint32_t w[8] = {x.x, x.y, x.z, x.w, y.x, y.y, y.z, y.w};
#pragma unroll
    for (int i = 0; i < 8; ++i) f[i] = __uint_as_float(w[i]);
}

// Channels c0 .. c0 + 7 of a row of K, turned.
template <typename E> __device__ __forceinline__ void packed_turn(const RopeArgs& a, const char* row, int c0, const double2* cs, float (&f)[8]) {
    const int rot = 2 * a.half;
    if (c0 >= rot) return;
    if (!a.halves) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            if (c0 + 2 * e >= rot) continue;
            const double2 z = cs[c0 / 2 + e];
            const double x = f[2 * e], y = f[2 * e + 1];
            f[2 * e] = packed_odd(x * z.x - y * z.y);
            f[2 * e + 1] = packed_odd(x * z.y + y * z.x);
        }
        return;
    }
    float g[8];
    if (a.half % 8 == 0) {
        packed_load((const E*)nullptr, row + (c0 < a.half ? c0 + a.half : c0 - a.half) * (int)sizeof(E), g);
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const int c = c0 + e;
            g[e] = c < rot ? RopeChunk<E>::load(row + (c < a.half ? c + a.half : c - a.half) * (int)sizeof(E)) : 0.0f;
        }
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const int c = c0 + e;
        if (c >= rot) continue;
        const bool first = c < a.half;
        const double2 z = cs[first ? c : c - a.half];
        f[e] = packed_odd(first ? f[e] * z.x - g[e] * z.y : g[e] * z.y + f[e] * z.x);
    }
}

// The least s with max < 7 * 2^(s - 127), from the largest magnitude's bits: a quarter on top of the mantissa carries from 1.75 on.
__device__ __forceinline__ uint32_t packed_scale(uint32_t top) {
    const int s = (int)((top + 0x200000u) >> 23) - 2;
    return (uint32_t)min(max(s, 2), 252);
}

// A workgroup takes up to 16 new rows of one sequence and some heads: of Q, which goes to q_out, or (from q_groups on) of K and V.  There
// d / 8 lanes take a row, eight channels each, four lanes a block of 32: its largest magnitude by two exchanges within the four, the
// codes by four conversions.  Everything is read and written once and the bytes bound it: 4680 rows of 12 heads of 128 are 94 MB with
// q_out, k_out and v_out, in 22.3 us (25 in the order of the caller's rows and with k_out and v_out by way of L2), and as fp32 180 MB in 35.9 (5.0 TB/s).
template <typename E, bool kChunks> __global__ __launch_bounds__(kRopeThreads) void packed_append_kernel(PackedAppendArgs a) {
    extern __shared__ __align__(16) char smem[];
    __shared__ int page_s[16];
    RowBlock rb;
    if (!block_of(a.c, 1, 1 << a.log_tb, a.per_seq, blockIdx.x, rb)) return;
    const int s = rb.seq, i0 = rb.block << a.log_tb;
    const SeqRows sr = rb.rows;
    const int n = min(min(sr.n, a.c.max_new) - i0, 1 << a.log_tb);
    const int row0 = sr.first + i0, p0 = sr.len - sr.n + i0, page_mask = (1 << a.c.log_page) - 1;
    const int32_t* pos = a.positions ? a.positions + (int64_t)row0 * a.rope.axes : nullptr;
    auto position = [&](int t, int axis) { return pos ? pos[t * a.rope.axes + axis] : p0 + t; };
    if ((int)blockIdx.y < a.q_groups) {
        float2* cs = reinterpret_cast<float2*>(smem);
        rope_angles(a.rope, n, position, cs);
        __syncthreads();
        const int h0 = blockIdx.y * a.hb, nh = min(a.hb, a.q_heads - h0);
        const RowAt at(a.order, a.log_tb, nh);
        rope_rows<E, kChunks>(a.rope, a.head_dim, a.units, at.rows(n), cs, [&](int r) {
            int t, h;
            at.find(r, t, h);
            RowMove m{nullptr, nullptr, t, a.rope.turns != nullptr};
            if (t >= n) return m;
            m.src = a.q + (row0 + t) * a.sq_n + (h + h0) * a.sq_h;
            m.dst = a.q_out + (row0 + t) * a.so_n + (h + h0) * a.so_h;
            return m;
        });
        return;
    }
    const int h0 = (blockIdx.y - a.q_groups) * a.hb, nh = min(a.hb, 2 * a.c.kv_heads - h0);
    double2* cs = reinterpret_cast<double2*>(smem);
    if ((int)threadIdx.x < n) {
        const int p = p0 + (int)threadIdx.x;
        const int id = p < 0 ? -1 : a.c.table[s * a.c.table_stride + (p >> a.c.log_page)];
        page_s[threadIdx.x] = id < a.c.pages ? id : -1;
    }
    if (h0 < a.c.kv_heads) packed_angles(a.rope, a.amplitude, n, position, cs);
    __syncthreads();
    const RowAt at(RowOrder{0}, a.log_tb, nh);   // the tokens of a head together: their codes and bytes are runs in its page
    const int width = a.head_dim / 8, u = threadIdx.x % width, rows = at.rows(n);
    for (int r = threadIdx.x / width; r < rows; r += kRopeThreads / width) {
        int t, h;
        at.find(r, t, h);
        h += h0;
        const bool is_v = h >= a.c.kv_heads;
        if (is_v) h -= a.c.kv_heads;
        const int id = t < n ? page_s[t] : -1;
        if (id < 0) continue;
        const char* row = is_v ? a.v + (row0 + t) * a.sv_n + h * a.sv_h : a.k + (row0 + t) * a.sk_n + h * a.sk_h;
        float f[8];
        packed_load((const E*)nullptr, row + 8 * u * (int)sizeof(E), f);
        if (!is_v && a.rope.turns) packed_turn<E>(a.rope, row, 8 * u, cs + t * a.rope.half, f);
        uint32_t top = 0;
#pragma unroll
        for (int e = 0; e < 8; ++e) top = max(top, __float_as_uint(f[e]) & 0x7fffffffu);
        top = max(top, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)top, 0xB1, 0xf, 0xf, false));   // lanes 1 0 3 2 of the four
        top = max(top, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)top, 0x4E, 0xf, 0xf, false));   // lanes 2 3 0 1
        const bool finite = top < 0x7f800000u;
        const uint32_t scale = finite ? packed_scale(top) : 255u;
        const float power = packed_power(scale);
        uint32_t w = 0;
        w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, f[0], f[1], power, 0);
        w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, f[2], f[3], power, 1);
        w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, f[4], f[5], power, 2);
        w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, f[6], f[7], power, 3);
        if (!finite) w = 0;
        const int slot = (p0 + t) & page_mask;
        char* dst = (is_v ? a.c.v : a.c.k) + id * a.c.page_b + h * a.head_b;
        *reinterpret_cast<uint32_t*>(dst + slot * (a.head_dim / 2) + 4 * u) = w;
        if (u % 4 == 0) dst[((int64_t)(a.head_dim / 2) << a.c.log_page) + slot * (a.head_dim / 32) + u / 4] = (char)scale;
        char* to = is_v ? a.v_out : a.k_out;
        if (!to) continue;
        to += is_v ? (row0 + t) * a.svo_n + h * a.svo_h : (row0 + t) * a.sko_n + h * a.sko_h;
        if constexpr (sizeof(E) == 2) {
            store_through(to + 16 * u, packed_bf16(w, power));
        } else {
            uint4 x[2];
            packed_f32(w, power, x);
            store_through(to + 32 * u, x[0]);
            store_through(to + 32 * u + 16, x[1]);
        }
    }
}

}  // namespace veda

extern "C" veda_status veda_packed_append(const veda_packed_cache* c, const veda_cache_batch* b, const void* k, veda_strides sk, const void* v,
                                          veda_strides sv, int32_t q_heads, const void* q, veda_strides sq, void* q_out, veda_strides sq_out,
                                          const veda_rope* rope, const int32_t* positions, void* k_out, veda_strides sk_out, void* v_out,
                                          veda_strides sv_out, void* stream) {
    veda_status st = veda::check_packed(c);
    if (st != VEDA_OK) return st;
    const veda_cache as = veda::packed_rows(c);
    st = veda::check_batch(&as, b);
    if (st != VEDA_OK) return st;
    if (q_heads < 0 || (q_heads == 0) != (q == nullptr) || (q_heads == 0) != (q_out == nullptr)) return VEDA_ERR_INVALID_ARG;
    if (rope && (rope->cfg.head_dim != c->head_dim || (!positions && rope->cfg.axes != 1))) return VEDA_ERR_INVALID_ARG;
    if (q_heads > 32 * 1024) return VEDA_ERR_UNSUPPORTED;
    if (b->seqs == 0 || b->rows == 0 || b->max_new == 0) return VEDA_OK;
    st = veda::check_rows(&as, b->rows, c->kv_heads, k, sk, false);
    if (st == VEDA_OK) st = veda::check_rows(&as, b->rows, c->kv_heads, v, sv, false);
    if (st == VEDA_OK && q_heads) st = veda::check_rows(&as, b->rows, q_heads, q, sq, false);
    if (st == VEDA_OK && q_heads) st = veda::check_rows(&as, b->rows, q_heads, q_out, sq_out, true);
    if (st == VEDA_OK && k_out) st = veda::check_rows(&as, b->rows, c->kv_heads, k_out, sk_out, true);
    if (st == VEDA_OK && v_out) st = veda::check_rows(&as, b->rows, c->kv_heads, v_out, sv_out, true);
    if (st != VEDA_OK) return st;
    if (q_heads && q == q_out && (sq.n != sq_out.n || sq.h != sq_out.h)) return VEDA_ERR_INVALID_ARG;
    for (const void* to : {k_out, v_out})      // rows are read by several lanes, and other workgroups
        if (to && (to == k || to == v || to == q || to == q_out)) return VEDA_ERR_INVALID_ARG;
    if (k_out && k_out == v_out) return VEDA_ERR_INVALID_ARG;
    if (rope) {
        int device = -1;
        VEDA_HIP_TRY(hipGetDevice(&device));
        if (device != rope->device) return VEDA_ERR_INVALID_ARG;
    }
    veda::PackedAppendArgs a;
    const int es = c->dtype == VEDA_BF16 ? 2 : 4, chunk = 16 / es, heads = q_heads + 2 * c->kv_heads;
    a.c = veda::packed_args(c, b);
    a.rope = veda::rope_args(rope, 0);
    a.amplitude = rope ? rope->amplitude : 1.0;
    a.q = (const char*)q; a.k = (const char*)k; a.v = (const char*)v;
    a.q_out = (char*)q_out; a.k_out = (char*)k_out; a.v_out = (char*)v_out;
    a.sq_h = sq.h * es; a.sq_n = sq.n * es; a.so_h = sq_out.h * es; a.so_n = sq_out.n * es;
    a.sk_h = sk.h * es; a.sk_n = sk.n * es; a.sv_h = sv.h * es; a.sv_n = sv.n * es;
    a.sko_h = sk_out.h * es; a.sko_n = sk_out.n * es; a.svo_h = sv_out.h * es; a.svo_n = sv_out.n * es;
    a.positions = positions;
    a.head_b = veda::packed_head_bytes(c);
    a.q_heads = q_heads; a.head_dim = c->head_dim;
    const bool chunks = veda::rope_in_chunks(a.rope, chunk);
    a.units = veda::rope_units(a.rope, c->head_dim, chunk, chunks);
    a.rope.through = veda::rope_whole_lines(a.rope, c->head_dim, es);
    veda::rope_blocks(a.c.max_new, b->seqs, heads, &a.log_tb, &a.hb);
    a.order = veda::row_order(sk.h < sk.n);
    a.q_groups = (q_heads + a.hb - 1) / a.hb;
    const int64_t each = ((int64_t)a.c.max_new + (1 << a.log_tb) - 1) >> a.log_tb, uniform = b->seqs * each;
    const int64_t gy = a.q_groups + (2 * c->kv_heads + a.hb - 1) / a.hb;
    int64_t gx = veda::block_items(b->seqs, b->rows, a.c.max_new, 1, (int64_t)1 << a.log_tb);
    a.per_seq = 0;
    if (veda::blocks_even(uniform, gx)) {
        gx = uniform;
        a.per_seq = (int32_t)each;
    }
    // a grid has less than 2^32 threads; and the search adds up 64 sequences' blocks in 32 bits
    if (gx >= 1 << 24 || gy > 65535 || each >= 1 << 24) return VEDA_ERR_UNSUPPORTED;
    const dim3 grid((unsigned)gx, (unsigned)gy);
    const size_t lds = (size_t)a.rope.half * sizeof(double2) << a.log_tb;
    const hipStream_t s = (hipStream_t)stream;
    if (c->dtype == VEDA_BF16 && chunks) hipLaunchKernelGGL((veda::packed_append_kernel<uint16_t, true>), grid, dim3(veda::kRopeThreads), lds, s, a);
    else if (c->dtype == VEDA_BF16) hipLaunchKernelGGL((veda::packed_append_kernel<uint16_t, false>), grid, dim3(veda::kRopeThreads), lds, s, a);
    else if (chunks) hipLaunchKernelGGL((veda::packed_append_kernel<uint32_t, true>), grid, dim3(veda::kRopeThreads), lds, s, a);
    else hipLaunchKernelGGL((veda::packed_append_kernel<uint32_t, false>), grid, dim3(veda::kRopeThreads), lds, s, a);
    return veda::launch_status("veda_packed_append");
}

extern "C" veda_status veda_packed_copy_pages(const veda_packed_cache* c, const int32_t* pairs, int64_t n, void* stream) {
    const veda_status st = veda::check_packed(c);
    if (st != VEDA_OK) return st;
    const veda::CacheArgs ca = veda::packed_args(c, nullptr);
    return veda::copy_pages(ca.k, ca.v, ca.page_b, c->kv_heads * veda::packed_head_bytes(c), c->pages, pairs, n, (hipStream_t)stream, "veda_packed_copy_pages");
}
