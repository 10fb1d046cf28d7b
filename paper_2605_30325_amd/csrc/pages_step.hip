// The page book on the GPU: a step's requests cut, evict and grow their sequences, and the page table, lengths, starts, positions and slots
// of the step's calls are written, without the host.
//
// Nothing is computed but numbers of pages: what costs time is how many dependent reads of memory and how many launches stand one behind
// the other.  Three kernels: a workgroup for each request looks whether it fits and gives back its pages (a long window leaves hundreds
// behind, read again at every step); one workgroup deals out the free pages, by sums over the requests and over the bits of the pages; and
// workgroups for each request and 1024 of its pages or rows write what comes out.
#include <algorithm>

#include "veda_internal.h"

namespace veda {

struct StepArgs {
    veda_device_pages book;
    veda_step step;
    veda_step_tables out;
};

__device__ __forceinline__ int step_pages(const StepArgs& a, int64_t tokens) { return (int)((tokens + a.book.page_tokens - 1) / a.book.page_tokens); }

// What request i asks of its sequence.
struct StepAsk {
    int seq, grow;
    int kept;                        // tokens that stay, or -1: refused
    int cut_from, cut_to;            // entries of the table that are given back
    int evict_from, evict_to;
};
// taken: an earlier request is about the same sequence.
__device__ __forceinline__ StepAsk step_ask(const StepArgs& a, int i, int seq, bool taken) {
    StepAsk k{seq, 0, -1, 0, 0, 0, 0};
    if (seq < 0 || seq >= a.book.max_seqs || taken) return k;
    const int64_t room = (int64_t)a.book.max_pages * a.book.page_tokens;
    const int64_t length = min((int64_t)max(a.book.length[seq], 0), room);
    const int64_t kept = a.step.keep ? min((int64_t)a.step.keep[i], length) : length;
    const int grow = a.step.grow[i], first = a.step.evict ? a.step.evict[2 * i] : 0, last = a.step.evict ? a.step.evict[2 * i + 1] : 0;
    if (kept < 0 || grow < 0 || grow > a.step.max_new || kept + grow > room || first < 0 || first > last || last > kept) return k;
    if (grow && kept % a.book.page_tokens) {
        const int open = a.book.table[(int64_t)seq * a.book.max_pages + kept / a.book.page_tokens];
        if (open < 0 || open >= a.book.pages) return k;
    }
    k.grow = grow;
    k.kept = (int)kept;
    k.cut_from = step_pages(a, kept);
    k.cut_to = step_pages(a, length);
    k.evict_from = step_pages(a, first);
    k.evict_to = last / a.book.page_tokens;
    return k;
}

constexpr int kGiveThreads = 256;

// A request's pages go back; kv_len[i] becomes what is kept, or -1.
__global__ __launch_bounds__(kGiveThreads) void pages_give_back_kernel(StepArgs a) {
    const int i = blockIdx.x, seq = a.step.seq ? a.step.seq[i] : i;
    bool taken = false;
    if (a.step.seq)
        for (int j = threadIdx.x; j < i; j += kGiveThreads) taken = taken || a.step.seq[j] == seq;
    taken = __syncthreads_or(taken);
    const StepAsk k = step_ask(a, i, seq, taken);
    if (threadIdx.x == 0) a.out.kv_len[i] = k.kept;
    int32_t* row = a.book.table + (int64_t)max(k.seq, 0) * a.book.max_pages;
    auto give = [&](int from, int to) {
        for (int x = from + (int)threadIdx.x; x < to; x += kGiveThreads) {
            const int id = row[x];
            if (id >= 0 && id < a.book.pages) atomicAnd(&a.book.used[id >> 5], ~(1u << (id & 31)));   // bits go in any order
            if (id != -1) row[x] = -1;
        }
    };
    give(k.cut_from, k.cut_to);
    give(k.evict_from, min(k.evict_to, k.cut_from));   // what is cut is gone already
}

constexpr int kDealThreads = 1024, kDealList = 4096;
struct Pair64 { int64_t pages, rows; };

// Sums over the threads before this one, and over all.  part: one entry a wave.
__device__ __forceinline__ Pair64 sums_before(Pair64 x, Pair64* part, Pair64& all) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    Pair64 up = x;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const int64_t p = __shfl_up((long long)up.pages, d), r = __shfl_up((long long)up.rows, d);
        if (lane >= d) { up.pages += p; up.rows += r; }
    }
    __syncthreads();
    if (lane == 63) part[wave] = up;
    __syncthreads();
    Pair64 before{0, 0};
    all = Pair64{0, 0};
    for (int w = 0; w < kDealThreads / 64; ++w) {
        if (w == wave) before = all;
        all.pages += part[w].pages;
        all.rows += part[w].rows;
    }
    return Pair64{before.pages + up.pages - x.pages, before.rows + up.rows - x.rows};
}

// Deals out the free pages.  Requests are served in their order while pages and rows suffice, so a sum over all before tells whether one is.
__global__ __launch_bounds__(kDealThreads) void pages_deal_kernel(StepArgs a) {
    extern __shared__ uint32_t deal_smem[];
    __shared__ Pair64 part[kDealThreads / 64];
    const int n = a.step.seqs, words = (a.book.pages + 31) / 32, tid = threadIdx.x;
    uint32_t* bits = deal_smem;                                      // [words]
    int* list = reinterpret_cast<int*>(bits + words);                // [kDealList] free pages in their order
    int* kept = list + kDealList;                                    // [n]
    int* start = kept + n;                                           // [n + 1] pages dealt out before a request
    for (int w = tid; w < words; w += kDealThreads) bits[w] = a.book.used[w];
    for (int i = tid; i < n; i += kDealThreads) kept[i] = a.out.kv_len[i];
    __syncthreads();
    // free pages of this thread's words, and before them
    const int each_w = (words + kDealThreads - 1) / kDealThreads, w0 = min(words, tid * each_w), w1 = min(words, w0 + each_w);
    auto free_of = [&](int w) {
        const int left = a.book.pages - 32 * w;
        return ~bits[w] & (left >= 32 ? 0xffffffffu : (1u << left) - 1u);
    };
    int mine = 0;
    for (int w = w0; w < w1; ++w) mine += __popc(free_of(w));
    Pair64 all;
    const int rank0 = (int)sums_before(Pair64{mine, 0}, part, all).pages;
    const int64_t pages_free = all.pages, rows_free = a.step.rows;
    // requests of this thread
    const int each = (n + kDealThreads - 1) / kDealThreads, i0 = min(n, tid * each), i1 = min(n, i0 + each);
    auto need = [&](int i) { return kept[i] < 0 ? 0 : step_pages(a, (int64_t)kept[i] + a.step.grow[i]) - step_pages(a, kept[i]); };
    Pair64 sum{0, 0};
    for (int i = i0; i < i1; ++i)
        if (kept[i] >= 0) {
            sum.pages += need(i);
            sum.rows += a.step.grow[i];
        }
    Pair64 at = sums_before(sum, part, all);
    // what the served ones get: the largest sums that still fit
    Pair64 top{0, 0}, x = at;
    for (int i = i0; i < i1; ++i) {
        if (kept[i] < 0) continue;
        x.pages += need(i);
        x.rows += a.step.grow[i];
        if (x.pages <= pages_free && x.rows <= rows_free) top = x;
    }
    __syncthreads();
#pragma unroll
    for (int d = 32; d >= 1; d >>= 1) {
        top.pages = max(top.pages, (int64_t)__shfl_xor((long long)top.pages, d));
        top.rows = max(top.rows, (int64_t)__shfl_xor((long long)top.rows, d));
    }
    if ((tid & 63) == 0) part[tid >> 6] = top;
    __syncthreads();
    for (int w = 0; w < kDealThreads / 64; ++w) {
        top.pages = max(top.pages, part[w].pages);
        top.rows = max(top.rows, part[w].rows);
    }
    for (int i = i0; i < i1; ++i) {
        const bool open = at.pages <= pages_free && at.rows <= rows_free;      // for all before
        start[i] = (int)(open ? at.pages : top.pages);
        a.out.q_start[i] = (int)(open ? at.rows : top.rows);
        int len = 0, status = VEDA_STEP_REFUSED;
        if (kept[i] >= 0) {
            const int grow = a.step.grow[i];
            at.pages += need(i);
            at.rows += grow;
            const bool served = at.pages <= pages_free && at.rows <= rows_free;
            len = kept[i] + (served ? grow : 0);
            status = served || grow == 0 ? VEDA_STEP_SERVED : VEDA_STEP_NO_ROOM;
            a.book.length[a.step.seq ? a.step.seq[i] : i] = len;
        }
        a.out.kv_len[i] = len;
        a.out.status[i] = status;
    }
    if (tid == 0) {
        start[n] = (int)top.pages;
        a.out.q_start[n] = (int)top.rows;
    }
    // the lowest free pages, kDealList at a time, to the requests
    const int dealt = (int)top.pages;
    for (int r0 = 0; r0 < dealt; r0 += kDealList) {
        const int r1 = min(dealt, r0 + kDealList);
        __syncthreads();
        if (rank0 < r1 && rank0 + mine > r0) {
            int rank = rank0;
            for (int w = w0; w < w1; ++w)
                for (uint32_t left = free_of(w); left; left &= left - 1, ++rank)
                    if (rank >= r0 && rank < r1) list[rank - r0] = 32 * w + __ffs((int)left) - 1;
        }
        __syncthreads();
        for (int r = r0 + tid; r < r1; r += kDealThreads) {
            int lo = 0, hi = n;                        // the last request that starts at r or before: the one that has it
            while (hi - lo > 1) {
                const int mid = (lo + hi) / 2;
                if (start[mid] <= r) lo = mid;
                else hi = mid;
            }
            const int seq = a.step.seq ? a.step.seq[lo] : lo;
            a.book.table[(int64_t)seq * a.book.max_pages + step_pages(a, kept[lo]) + r - start[lo]] = list[r - r0];
        }
    }
    // and their bits
    for (int w = w0, rank = rank0; w < w1 && rank < dealt; ++w) {
        uint32_t taken = 0;
        for (uint32_t left = free_of(w); left && rank < dealt; left &= left - 1, ++rank) taken |= left & (0u - left);
        if (taken) a.book.used[w] = bits[w] | taken;
    }
}

constexpr int kWriteThreads = 256, kWriteItems = 1024, kWriteMost = 64;    // items of a workgroup, workgroups of a request

// Request blockIdx.x: entries of its row of the page table, and its rows.
__global__ __launch_bounds__(kWriteThreads) void pages_write_kernel(StepArgs a) {
    const int i = blockIdx.x, len = a.out.kv_len[i], row0 = a.out.q_start[i], added = a.out.q_start[i + 1] - row0;
    const int seq = a.step.seq ? a.step.seq[i] : i, have = step_pages(a, len);
    const int32_t* from = a.book.table + (int64_t)(have ? seq : 0) * a.book.max_pages;       // a refused one has no pages
    int32_t* to = a.out.page_table + i * a.out.table_stride;
    const int64_t x0 = (int64_t)blockIdx.y * kWriteThreads + threadIdx.x, step = (int64_t)gridDim.y * kWriteThreads;
    for (int64_t x = x0; x < a.book.max_pages; x += step) to[x] = x < have ? from[x] : -1;
    for (int64_t r = x0; r < added; r += step) {
        const int p = len - added + (int)r;
        const int64_t row = row0 + r;
        if (a.out.positions) {
            if (a.step.axes == 1) {
                a.out.positions[row] = p;
            } else {
                const int line = p / a.step.frame_w;
                a.out.positions[3 * row] = line / a.step.frame_h;
                a.out.positions[3 * row + 1] = line % a.step.frame_h;
                a.out.positions[3 * row + 2] = p % a.step.frame_w;
            }
        }
        if (a.out.row_seq) a.out.row_seq[row] = i;
        if (a.out.slots) a.out.slots[row] = (int64_t)from[p / a.book.page_tokens] * a.book.page_tokens + p % a.book.page_tokens;
    }
}

}  // namespace veda

extern "C" veda_status veda_pages_step(const veda_device_pages* book, const veda_step* step, const veda_step_tables* out, void* stream) {
    if (!book || !step || !out) return VEDA_ERR_INVALID_ARG;
    if (book->pages < 1 || book->page_tokens < 1 || book->max_seqs < 1 || book->max_pages < 1 || !book->table || !book->length || !book->used) return VEDA_ERR_INVALID_ARG;
    if (step->seqs < 0 || step->rows < 0 || step->max_new < 0 || (step->axes != 1 && step->axes != 3)) return VEDA_ERR_INVALID_ARG;
    if (step->axes == 3 && (step->frame_h < 1 || step->frame_w < 1)) return VEDA_ERR_INVALID_ARG;
    if (!out->q_start || out->table_stride < book->max_pages) return VEDA_ERR_INVALID_ARG;
    if (step->seqs > 0 && (!step->grow || !out->page_table || !out->kv_len || !out->status)) return VEDA_ERR_INVALID_ARG;
    if (!step->seq && step->seqs > book->max_seqs) return VEDA_ERR_INVALID_ARG;
    for (const int32_t* in : {step->seq, step->keep, step->evict, step->grow})       // read after others' results are written
        for (const int32_t* res : {out->page_table, out->kv_len, out->q_start, out->status, out->positions, out->row_seq, book->table, book->length})
            if (in && in == res) return VEDA_ERR_INVALID_ARG;
    if (book->pages > 1 << 19 || book->max_seqs > 8192 || step->seqs > 8192 || step->rows > 1 << 30) return VEDA_ERR_UNSUPPORTED;
    if ((int64_t)book->max_pages * book->page_tokens > (int64_t)1 << 30) return VEDA_ERR_UNSUPPORTED;
    const hipStream_t s = (hipStream_t)stream;
    const veda::StepArgs a{*book, *step, *out};
    const unsigned n = (unsigned)step->seqs;
    veda_status st = VEDA_OK;
    if (n) {
        hipLaunchKernelGGL(veda::pages_give_back_kernel, dim3(n), dim3(veda::kGiveThreads), 0, s, a);
        st = veda::launch_status("veda_pages_step");
        if (st != VEDA_OK) return st;
    }
    const size_t lds = 4 * ((size_t)(book->pages + 31) / 32 + veda::kDealList + 2 * (size_t)n + 1);
    if (lds > 64 * 1024) VEDA_HIP_TRY(hipFuncSetAttribute((const void*)veda::pages_deal_kernel, hipFuncAttributeMaxDynamicSharedMemorySize, 160 * 1024 - 512));
    hipLaunchKernelGGL(veda::pages_deal_kernel, dim3(1), dim3(veda::kDealThreads), lds, s, a);
    st = veda::launch_status("veda_pages_step");
    if (st != VEDA_OK || !n) return st;
    const int64_t widest = std::max<int64_t>(book->max_pages, std::min(step->max_new, step->rows));
    hipLaunchKernelGGL(veda::pages_write_kernel, dim3(n, (unsigned)std::min<int64_t>(veda::kWriteMost, (widest + veda::kWriteItems - 1) / veda::kWriteItems)), dim3(veda::kWriteThreads), 0, s, a);
    return veda::launch_status("veda_pages_step");
}
