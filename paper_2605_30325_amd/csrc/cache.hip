// The paged cache: checks, appending the newest rows, copies of pages.
#include "cache.h"
#include "rope_rows.h"
#include "rows_apart.h"

namespace veda {

veda_status check_cache(const veda_cache* c) {
    if (!c || !c->k || !c->v || c->pages < 1 || c->kv_heads < 1 || c->page_stride < 0) return VEDA_ERR_INVALID_ARG;
    if (c->dtype != VEDA_F32 && c->dtype != VEDA_BF16) return VEDA_ERR_INVALID_ARG;
    if (c->head_dim != 64 && c->head_dim != 128) return VEDA_ERR_UNSUPPORTED;
    if (c->kv_heads > 1024) return VEDA_ERR_UNSUPPORTED;
    if (c->page_tokens < 16 || c->page_tokens > 256 || (c->page_tokens & (c->page_tokens - 1))) return VEDA_ERR_UNSUPPORTED;
    const int64_t elems = (int64_t)c->kv_heads * c->page_tokens * c->head_dim, es = c->dtype == VEDA_BF16 ? 2 : 4;
    if (c->page_stride && c->page_stride < elems) return VEDA_ERR_INVALID_ARG;
    if ((c->page_stride * es) % 16 || !aligned16(c->k) || !aligned16(c->v)) return VEDA_ERR_UNSUPPORTED;
    return VEDA_OK;
}

veda_status check_batch(const veda_cache* c, const veda_cache_batch* b) {
    if (!b || b->seqs < 0 || b->rows < 0 || b->max_new < 0 || b->max_pages < 1 || b->table_stride < b->max_pages) return VEDA_ERR_INVALID_ARG;
    if (b->seqs > 0 && (!b->page_table || !b->kv_len || !b->q_start)) return VEDA_ERR_INVALID_ARG;
    if ((int64_t)b->max_pages * c->page_tokens > (int64_t)1 << 30 || b->rows > 1 << 30) return VEDA_ERR_UNSUPPORTED;
    return VEDA_OK;
}

CacheArgs cache_args(const veda_cache* c, const veda_cache_batch* b) {
    CacheArgs a{};
    const int es = c->dtype == VEDA_BF16 ? 2 : 4;
    a.k = (char*)c->k; a.v = (char*)c->v;
    a.page_b = es * (c->page_stride ? c->page_stride : (int64_t)c->kv_heads * c->page_tokens * c->head_dim);
    a.pages = c->pages; a.kv_heads = c->kv_heads;
    for (a.log_page = 4; 1 << a.log_page < c->page_tokens; ++a.log_page) {}
    if (b) {
        a.table = b->page_table; a.kv_len = b->kv_len; a.q_start = b->q_start;
        a.table_stride = b->table_stride;
        a.seqs = b->seqs; a.rows = b->rows; a.max_pages = b->max_pages;
        a.max_new = b->max_new < b->rows ? b->max_new : b->rows;
    }
    return a;
}

veda_status check_rows(const veda_cache* c, int32_t rows, int32_t heads, const void* p, veda_strides& s, bool distinct) {
    const int es = c->dtype == VEDA_BF16 ? 2 : 4, d = c->head_dim;
    if (rows == 1) s.n = 0;
    if (heads == 1) s.h = 0;
    if (!p || s.h < 0 || s.n < 0) return VEDA_ERR_INVALID_ARG;
    if (distinct) {
        const RowsApart apart = rows_apart({rows, s.n}, {heads, s.h}, {1, 0}, d);
        if (apart != RowsApart::kApart) return apart == RowsApart::kShare ? VEDA_ERR_INVALID_ARG : VEDA_ERR_UNSUPPORTED;
    }
    if (!aligned16(p) || (s.h * es) % 16 || (s.n * es) % 16) return VEDA_ERR_UNSUPPORTED;
    return VEDA_OK;
}

struct AppendArgs {
    CacheArgs c;
    RopeArgs rope;
    const char *q, *k, *v;
    char* q_out;
    int64_t sq_h, sq_n, so_h, so_n, sk_h, sk_n, sv_h, sv_n;   // bytes
    const int32_t* positions;   // null: the position in the sequence
    int32_t q_heads, head_dim, units, log_tb, hb, per_seq;
    RowOrder order;
};

// A workgroup takes up to 16 new rows of one sequence and some of the heads of Q, K and V (numbered one behind the other): Q goes to
// q_out, K and V to the rows' slots.  Everything is read and written once, 16 bytes at a time, in runs of a row.
template <typename E, bool kChunks> __global__ __launch_bounds__(kRopeThreads) void append_kernel(AppendArgs a) {
    extern __shared__ float2 cs[];
    __shared__ int page_s[16];
    RowBlock rb;
    if (!block_of(a.c, 1, 1 << a.log_tb, a.per_seq, blockIdx.x, rb)) return;
    const int s = rb.seq, i0 = rb.block << a.log_tb;
    const SeqRows sr = rb.rows;
    const int n = min(min(sr.n, a.c.max_new) - i0, 1 << a.log_tb);
    const int row0 = sr.first + i0, p0 = sr.len - sr.n + i0, page_mask = (1 << a.c.log_page) - 1;
    if ((int)threadIdx.x < n) {
        const int p = p0 + (int)threadIdx.x;
        const int id = p < 0 ? -1 : a.c.table[s * a.c.table_stride + (p >> a.c.log_page)];
        page_s[threadIdx.x] = id < a.c.pages ? id : -1;
    }
    const int32_t* pos = a.positions ? a.positions + (int64_t)row0 * a.rope.axes : nullptr;
    rope_angles(a.rope, n, [&](int t, int axis) { return pos ? pos[t * a.rope.axes + axis] : p0 + t; }, cs);
    __syncthreads();
    const int heads = a.q_heads + 2 * a.c.kv_heads, h0 = blockIdx.y * a.hb, nh = min(a.hb, heads - h0);
    const int64_t row_b = (int64_t)a.head_dim * sizeof(E), head_b = row_b << a.c.log_page;
    const RowAt at(a.order, a.log_tb, nh);
    rope_rows<E, kChunks>(a.rope, a.head_dim, a.units, at.rows(n), cs,
                          [&](int r) {
                              int t, h;
                              at.find(r, t, h);
                              h += h0;
                              RowMove m{nullptr, nullptr, t, a.rope.turns != nullptr};
                              if (t >= n) return m;
                              if (h < a.q_heads) {
                                  m.src = a.q + (row0 + t) * a.sq_n + h * a.sq_h;
                                  m.dst = a.q_out + (row0 + t) * a.so_n + h * a.so_h;
                                  return m;
                              }
                              h -= a.q_heads;
                              const bool is_v = h >= a.c.kv_heads;
                              if (is_v) { h -= a.c.kv_heads; m.turn = false; }
                              const int id = page_s[t];
                              if (id < 0) return m;
                              m.src = is_v ? a.v + (row0 + t) * a.sv_n + h * a.sv_h : a.k + (row0 + t) * a.sk_n + h * a.sk_h;
                              m.dst = (is_v ? a.c.v : a.c.k) + id * a.c.page_b + h * head_b + ((p0 + t) & page_mask) * row_b;
                              return m;
                          });
}

// Pairs of one launch, by value: no list in device memory that a later call could overwrite before this one has run.  Arguments
// are copied on the host at every launch, so short lists (a branch's open page) have a form of their own: 3.6 KB against 256 bytes.
constexpr int kCopyPairs = 448, kCopyPairsShort = 28;
template <int N> struct CopyArgs {
    char *k, *v;
    int64_t page_b;
    int32_t chunks;              // 16-byte chunks of a page
    int32_t pair[N][2];
};

// A copy: 4 bytes moved for each byte of a page, nothing computed.  Stores go past the die's L2: kept there, they cost 50 us instead of 17
// for 1000 pages of 16 KB, and 180 instead of 152 us (5.2 TB/s) for 1000 pages of 192 KB; two chunks a thread, four and eight are 3 % slower.
constexpr int kCopyChunks = 2;   // 16-byte chunks in flight per thread

template <int N> __global__ __launch_bounds__(256) void copy_pages_kernel(CopyArgs<N> a) {
    char* pool = blockIdx.z ? a.v : a.k;
    const uint4* src = reinterpret_cast<const uint4*>(pool + a.pair[blockIdx.y][0] * a.page_b);
    uint4* dst = reinterpret_cast<uint4*>(pool + a.pair[blockIdx.y][1] * a.page_b);
    const int c0 = blockIdx.x * (256 * kCopyChunks) + threadIdx.x;
    uint4 x[kCopyChunks];
#pragma unroll
    for (int j = 0; j < kCopyChunks; ++j)
        if (c0 + j * 256 < a.chunks) x[j] = src[c0 + j * 256];
#pragma unroll
    for (int j = 0; j < kCopyChunks; ++j)
        if (c0 + j * 256 < a.chunks) store_through(dst + c0 + j * 256, x[j]);
}

}  // namespace veda

extern "C" veda_status veda_cache_append(const veda_cache* c, const veda_cache_batch* b, const void* k, veda_strides sk, const void* v,
                                         veda_strides sv, int32_t q_heads, const void* q, veda_strides sq, void* q_out,
                                         veda_strides sq_out, const veda_rope* rope, const int32_t* positions, void* stream) {
    veda_status st = veda::check_cache(c);
    if (st == VEDA_OK) st = veda::check_batch(c, b);
    if (st != VEDA_OK) return st;
    if (q_heads < 0 || (q_heads == 0) != (q == nullptr) || (q_heads == 0) != (q_out == nullptr)) return VEDA_ERR_INVALID_ARG;
    if (rope && (rope->cfg.head_dim != c->head_dim || (!positions && rope->cfg.axes != 1))) return VEDA_ERR_INVALID_ARG;
    if (q_heads > 32 * 1024) return VEDA_ERR_UNSUPPORTED;
    if (b->seqs == 0 || b->rows == 0 || b->max_new == 0) return VEDA_OK;
    st = veda::check_rows(c, b->rows, c->kv_heads, k, sk, false);
    if (st == VEDA_OK) st = veda::check_rows(c, b->rows, c->kv_heads, v, sv, false);
    if (st == VEDA_OK && q_heads) st = veda::check_rows(c, b->rows, q_heads, q, sq, false);
    if (st == VEDA_OK && q_heads) st = veda::check_rows(c, b->rows, q_heads, q_out, sq_out, true);
    if (st != VEDA_OK) return st;
    if (q_heads && q == q_out && (sq.n != sq_out.n || sq.h != sq_out.h)) return VEDA_ERR_INVALID_ARG;
    if (rope) {
        int device = -1;
        VEDA_HIP_TRY(hipGetDevice(&device));
        if (device != rope->device) return VEDA_ERR_INVALID_ARG;
    }
    veda::AppendArgs a;
    const int es = c->dtype == VEDA_BF16 ? 2 : 4, chunk = 16 / es, heads = q_heads + 2 * c->kv_heads;
    a.c = veda::cache_args(c, b);
    a.rope = veda::rope_args(rope, 0);
    a.q = (const char*)q; a.k = (const char*)k; a.v = (const char*)v; a.q_out = (char*)q_out;
    a.sq_h = sq.h * es; a.sq_n = sq.n * es; a.so_h = sq_out.h * es; a.so_n = sq_out.n * es;
    a.sk_h = sk.h * es; a.sk_n = sk.n * es; a.sv_h = sv.h * es; a.sv_n = sv.n * es;
    a.positions = positions;
    a.q_heads = q_heads; a.head_dim = c->head_dim;
    const bool chunks = veda::rope_in_chunks(a.rope, chunk);
    a.units = veda::rope_units(a.rope, c->head_dim, chunk, chunks);
    a.rope.through = veda::rope_whole_lines(a.rope, c->head_dim, es);
    veda::rope_blocks(a.c.max_new, b->seqs, heads, &a.log_tb, &a.hb);
    a.order = veda::row_order(sk.h < sk.n);
    const int64_t each = ((int64_t)a.c.max_new + (1 << a.log_tb) - 1) >> a.log_tb, uniform = b->seqs * each, gy = (heads + a.hb - 1) / a.hb;
    int64_t gx = veda::block_items(b->seqs, b->rows, a.c.max_new, 1, (int64_t)1 << a.log_tb);
    a.per_seq = 0;
    if (veda::blocks_even(uniform, gx)) {
        gx = uniform;
        a.per_seq = (int32_t)each;
    }
    // a grid has less than 2^32 threads; and the search adds up 64 sequences' blocks in 32 bits
    if (gx >= 1 << 24 || gy > 65535 || each >= 1 << 24) return VEDA_ERR_UNSUPPORTED;
    const dim3 grid((unsigned)gx, (unsigned)gy);
    const size_t lds = (size_t)a.rope.half * sizeof(float2) << a.log_tb;
    const hipStream_t s = (hipStream_t)stream;
    if (c->dtype == VEDA_BF16 && chunks) hipLaunchKernelGGL((veda::append_kernel<uint16_t, true>), grid, dim3(veda::kRopeThreads), lds, s, a);
    else if (c->dtype == VEDA_BF16) hipLaunchKernelGGL((veda::append_kernel<uint16_t, false>), grid, dim3(veda::kRopeThreads), lds, s, a);
    else if (chunks) hipLaunchKernelGGL((veda::append_kernel<uint32_t, true>), grid, dim3(veda::kRopeThreads), lds, s, a);
    else hipLaunchKernelGGL((veda::append_kernel<uint32_t, false>), grid, dim3(veda::kRopeThreads), lds, s, a);
    return veda::launch_status("veda_cache_append");
}

extern "C" veda_status veda_cache_copy_pages(const veda_cache* c, const int32_t* pairs, int64_t n, void* stream) {
    veda_status st = veda::check_cache(c);
    if (st != VEDA_OK) return st;
    if (n < 0 || (n > 0 && !pairs)) return VEDA_ERR_INVALID_ARG;
    for (int64_t i = 0; i < 2 * n; ++i)
        if (pairs[i] < 0 || pairs[i] >= c->pages) return VEDA_ERR_INVALID_ARG;
    if (n == 0) return VEDA_OK;
    const veda::CacheArgs ca = veda::cache_args(c, nullptr);
    veda::CopyArgs<veda::kCopyPairs> a;
    a.k = ca.k; a.v = ca.v; a.page_b = ca.page_b;
    a.chunks = (int32_t)((int64_t)c->kv_heads * c->page_tokens * c->head_dim * (c->dtype == VEDA_BF16 ? 2 : 4) / 16);
    const unsigned gx = (unsigned)((a.chunks + 256 * veda::kCopyChunks - 1) / (256 * veda::kCopyChunks));
    const hipStream_t s = (hipStream_t)stream;
    // A launch ends where the next pair touches what its pairs write, or writes what they read: stream order then gives the
    // order of the list.  Long lists keep a note for every page (bit 0 read, bit 1 written by the open launch), short ones look back.
    std::vector<uint8_t> note;
    if (n > veda::kCopyPairsShort) {
        try {
            note.assign((size_t)c->pages, 0);
        } catch (const std::exception&) {
            return veda::hip_fail(hipErrorOutOfMemory, "veda_cache_copy_pages");
        }
    }
    int m = 0;
    auto launch = [&]() -> veda_status {
        if (m == 0) return VEDA_OK;
        if (m <= veda::kCopyPairsShort) {
            veda::CopyArgs<veda::kCopyPairsShort> b;
            b.k = a.k; b.v = a.v; b.page_b = a.page_b; b.chunks = a.chunks;
            for (int i = 0; i < veda::kCopyPairsShort; ++i)
                for (int j = 0; j < 2; ++j) b.pair[i][j] = i < m ? a.pair[i][j] : 0;
            hipLaunchKernelGGL((veda::copy_pages_kernel<veda::kCopyPairsShort>), dim3(gx, (unsigned)m, 2), dim3(256), 0, s, b);
        } else {
            hipLaunchKernelGGL((veda::copy_pages_kernel<veda::kCopyPairs>), dim3(gx, (unsigned)m, 2), dim3(256), 0, s, a);
        }
        if (!note.empty())
            for (int i = 0; i < m; ++i) note[a.pair[i][0]] = note[a.pair[i][1]] = 0;
        m = 0;
        return veda::launch_status("veda_cache_copy_pages");
    };
    for (int64_t i = 0; i < n; ++i) {
        const int32_t from = pairs[2 * i], to = pairs[2 * i + 1];
        if (from == to) continue;
        bool touches = m == veda::kCopyPairs;
        if (!note.empty()) touches = touches || (note[from] & 2) || note[to];
        else
            for (int j = 0; j < m; ++j) touches = touches || a.pair[j][1] == from || a.pair[j][1] == to || a.pair[j][0] == to;
        if (touches) {
            st = launch();
            if (st != VEDA_OK) return st;
        }
        a.pair[m][0] = from;
        a.pair[m][1] = to;
        ++m;
        if (!note.empty()) {
            note[from] |= 1;
            note[to] |= 2;
        }
    }
    return launch();
}
