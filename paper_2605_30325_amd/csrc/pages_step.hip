// The page book on the GPU: a step's requests cut, evict and grow their sequences, and the page table, lengths, starts, positions and slots
// of the step's calls are written, without the host.
//
// Nothing is computed but numbers of pages: what costs time is how many dependent reads of memory and how many launches stand one behind
// the other.  Where little is written one workgroup does it all, with the requests, the dealt pages and the table's entries in LDS and registers
// (64 requests of 126 pages: 7 us instead of 16 for the three kernels below).  Otherwise: a workgroup for each request looks whether it fits and
// gives back its pages (a long window leaves hundreds behind, read again at every step); one workgroup deals out the free pages, by sums over the
// requests and over the bits of the pages; and workgroups for each request write what comes out.
#include <algorithm>

#include "cache.h"

namespace veda {

struct StepArgs {
    veda_device_pages book;
    veda_step step;
    veda_step_tables out;
    // t / page_tokens = t * magic >> shift for t < 2^31, without a branch for powers of two: 2^(shift - 31) is the least power of two from page_tokens on,
    // magic = ceil(2^shift / page_tokens) less than 1 too much, so the quotient less than 2^31 / 2^shift <= 1 / page_tokens, which its floor does not show.
    uint32_t magic;
    int32_t shift;
};

// Whole pages in 0 .. 2^31 tokens, and pages of 0 .. 2^30 tokens.
__device__ __forceinline__ int step_whole(const StepArgs& a, uint32_t tokens) { return (int)((uint64_t)tokens * a.magic >> a.shift); }
__device__ __forceinline__ int step_pages(const StepArgs& a, int tokens) { return step_whole(a, (uint32_t)tokens + (uint32_t)a.book.page_tokens - 1u); }

// What request i asks of its sequence.
struct StepAsk {
    int seq, grow;
    int kept;                        // tokens that stay, or -1: refused
    int open;                        // the page that the next token falls into, if it has tokens already
    int cut_from, cut_to;            // entries of the table that are given back
    int evict_from, evict_to;
};
// taken: an earlier request is about the same sequence.
__device__ __forceinline__ StepAsk step_ask(const StepArgs& a, int i, int seq, bool taken) {
    StepAsk k{seq, 0, -1, -1, 0, 0, 0, 0};
    if (seq < 0 || seq >= a.book.max_seqs || taken) return k;
    const int room = a.book.max_pages * a.book.page_tokens;      // up to 2^30
    const int length = min(max(a.book.length[seq], 0), room), kept = a.step.keep ? min(a.step.keep[i], length) : length;
    const int grow = a.step.grow[i], first = a.step.evict ? a.step.evict[2 * i] : 0, last = a.step.evict ? a.step.evict[2 * i + 1] : 0;
    if (kept < 0 || grow < 0 || grow > a.step.max_new || grow > room - kept || first < 0 || first > last || last > kept) return k;
    k.cut_from = step_pages(a, kept);
    if (grow && k.cut_from * a.book.page_tokens > kept) {
        k.open = a.book.table[(int64_t)seq * a.book.max_pages + k.cut_from - 1];
        if (k.open < 0 || k.open >= a.book.pages) return k;
    }
    k.grow = grow;
    k.kept = kept;
    k.cut_to = step_pages(a, length);
    k.evict_from = step_pages(a, first);
    k.evict_to = step_whole(a, (uint32_t)last);
    return k;
}

constexpr int kGiveThreads = 256;

// A request's pages go back; its sequence's length becomes what is kept, and status[i] whether it is refused.
__global__ __launch_bounds__(kGiveThreads) void pages_give_back_kernel(StepArgs a) {
    const int i = blockIdx.x, seq = a.step.seq ? a.step.seq[i] : i;
    bool taken = false;
    if (a.step.seq)
        for (int j = threadIdx.x; j < i; j += kGiveThreads) taken = taken || a.step.seq[j] == seq;
    taken = __syncthreads_or(taken);
    const StepAsk k = step_ask(a, i, seq, taken);
    __syncthreads();    // all threads have read the length
    if (threadIdx.x == 0) {
        a.out.status[i] = k.kept < 0 ? VEDA_STEP_REFUSED : VEDA_STEP_SERVED;
        if (k.kept >= 0) a.book.length[k.seq] = k.kept;
    }
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

constexpr int kDealThreads = 1024, kDealWaves = kDealThreads / 64;
constexpr int kStepLds = 158 * 1024;    // of a launch, beside what the kernels have by themselves

// Sums over the threads before this one, and over all, of N numbers.
template <int N> __device__ __forceinline__ void sums_before(const int (&x)[N], int (*part)[kDealWaves], int (&before)[N], int (&all)[N]) {
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    int up[N];
#pragma unroll
    for (int j = 0; j < N; ++j) {
        up[j] = lanes_up_to(x[j]);
        if (lane == 63) part[j][wave] = up[j];
    }
    __syncthreads();
#pragma unroll
    for (int j = 0; j < N; ++j) {
        const int w = lane < kDealWaves ? part[j][lane] : 0, to = lanes_up_to(w);
        before[j] = __builtin_amdgcn_readlane(to, wave) - __builtin_amdgcn_readlane(w, wave) + up[j] - x[j];
        all[j] = __builtin_amdgcn_readlane(to, 63);
    }
}
// The largest of a number that no later thread has a smaller one of (but 0: none), into `top`.  One lane of a wave speaks for all: 64 that
// change the same word of LDS wait for each other, 2 us.
__device__ __forceinline__ void last_of(int* top, int x) {
    const uint64_t some = __ballot(x != 0);
    if (some && (int)(threadIdx.x & 63) == 63 - __clzll((long long)some)) atomicMax(top, x);
}
// Free pages of word w of the bits.
__device__ __forceinline__ uint32_t step_free(const StepArgs& a, int w, uint32_t used) {
    const int left = a.book.pages - 32 * w;
    return ~used & (left >= 32 ? 0xffffffffu : (1u << left) - 1u);
}

// Deals out the free pages, the lowest first: entries of the book's table, and q_start and kv_len.  A request is served if the sums of pages and rows
// up to it fit (and so do all before it).  Every workgroup forms all sums, and takes every so manieth eight of the bits (the bits are set by the next
// kernel, when all have been counted): 17,000 scattered entries for 700 requests, out of 480,000 pages, 12 us (17 with a word to a thread and all
// threads' sums into one word of LDS, 21 by one workgroup).
__global__ __launch_bounds__(kDealThreads) void pages_deal_kernel(StepArgs a) {
    extern __shared__ int deal_smem[];
    constexpr int kParts = 4 * 64;                                   // sums of 64 words: one of every wave for 1024
    __shared__ int part[4][kDealWaves];
    __shared__ __align__(16) int part_w[kParts];
    __shared__ int top_s[2];
    const int n = a.step.seqs, words = (a.book.pages + 31) / 32, tid = threadIdx.x;
    int* rank = deal_smem;                                           // [words] the bits, then free pages before those of a word
    int* have = rank + words;                                        // [n] pages that a request's sequence keeps
    int* start = have + n;                                           // [n + 1] pages that it needs, then those dealt out before
    uint16_t* seq_s = reinterpret_cast<uint16_t*>(start + n + 1);    // [n]
    const int lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int each = (n + kDealThreads - 1) / kDealThreads, i0 = min(n, tid * each), i1 = min(n, i0 + each);
    // Every read is the first since another kernel wrote, 1-2 us: as few of them as can be stand one behind the other.
    const bool one = i0 < i1;
    const int status0 = one ? a.out.status[i0] : VEDA_STEP_REFUSED, seq0 = one ? a.step.seq ? a.step.seq[i0] : i0 : 0, grow0 = one ? a.step.grow[i0] : 0;
    if (tid < kParts) part_w[tid] = 0;
    if (tid < 2) top_s[tid] = 0;
#pragma unroll 8
    for (int w = tid; w < words; w += kDealThreads) rank[w] = (int)a.book.used[w];
    // Pages and rows of the thread's requests.  Sums of 8192 numbers up to 2^30 come in two parts.
    int sum[4] = {0, 0, 0, 0}, before[4], all[4];
#pragma unroll 1
    for (int i = i0; i < i1; ++i) {
        int need = 0, pages = -1;
        if ((i == i0 ? status0 : a.out.status[i]) != VEDA_STEP_REFUSED) {
            const int seq = i == i0 ? seq0 : a.step.seq ? a.step.seq[i] : i, kept = a.book.length[seq], grow = i == i0 ? grow0 : a.step.grow[i];
            seq_s[i] = (uint16_t)seq;
            pages = step_pages(a, kept);
            need = step_pages(a, kept + grow) - pages;
            sum[0] += need & 0x7fff; sum[1] += need >> 15;
            sum[2] += grow & 0x7fff; sum[3] += grow >> 15;
        }
        have[i] = pages;                                             // -1: refused
        start[i] = need;
    }
    __syncthreads();
    // Free pages: sums within 64 words, then of those, four to a lane.
#pragma unroll 1
    for (int w0 = wave * 64; w0 < words; w0 += kDealThreads) {
        const int w = w0 + lane, own = w < words ? __popc(step_free(a, w, (uint32_t)rank[w])) : 0, up = lanes_up_to(own);
        if (w < words) rank[w] = up - own;
        if (lane == 63) part_w[w0 / 64] = up;
    }
    sums_before(sum, part, before, all);
    int4 of = reinterpret_cast<const int4*>(part_w)[lane];
    const int to = lanes_up_to(of.x + of.y + of.z + of.w), pages_free = __builtin_amdgcn_readlane(to, 63);
    of.w = to - of.w;                                                // what lies before each of the four
    of.z = of.w - of.z;
    of.y = of.z - of.y;
    of.x = of.y - of.x;
    __syncthreads();
    if (wave == 0) reinterpret_cast<int4*>(part_w)[lane] = of;
    int64_t pages = ((int64_t)before[1] << 15) + before[0], rows = ((int64_t)before[3] << 15) + before[2];
    auto fits = [&](int64_t pages, int64_t rows) { return pages <= pages_free && rows <= a.step.rows; };
    {
        int64_t p = pages, r = rows;
        int top[2] = {0, 0};
#pragma unroll 1
        for (int i = i0; i < i1; ++i) {
            p += start[i];
            r += have[i] < 0 ? 0 : i == i0 ? grow0 : a.step.grow[i];
            if (fits(p, r)) {
                top[0] = (int)p;
                top[1] = (int)r;
            }
        }
        last_of(&top_s[0], top[0]);
        last_of(&top_s[1], top[1]);
    }
    __syncthreads();
    const int dealt = top_s[0];
#pragma unroll 1
    for (int w = tid; w < words; w += kDealThreads) rank[w] += part_w[w / 64];
#pragma unroll 1
    for (int i = i0; i < i1; ++i) {
        const bool open = fits(pages, rows), asks = have[i] >= 0;    // open: there is room for all before
        const int need = start[i], grow = !asks ? 0 : i == i0 ? grow0 : a.step.grow[i];
        start[i] = open ? (int)pages : dealt;
        const int at = open ? (int)rows : top_s[1];
        pages += need;
        rows += grow;
        if (blockIdx.x == 0) {
            a.out.q_start[i] = at;
            a.out.kv_len[i] = asks ? a.book.length[seq_s[i]] + (fits(pages, rows) ? grow : 0) : 0;
        }
    }
    if (tid == 0) {
        start[n] = dealt;
        if (blockIdx.x == 0) a.out.q_start[n] = top_s[1];
    }
    __syncthreads();
    for (int x = tid * gridDim.x + blockIdx.x;; x += kDealThreads * gridDim.x) {      // eight pages
        const int w = x / 4, shift = 8 * (x & 3);
        if (w >= words || rank[w] >= dealt) break;                                    // ranks only grow
        uint32_t left = step_free(a, w, a.book.used[w]);
        int r = rank[w] + __popc(left & ((1u << shift) - 1u));
        left &= 0xffu << shift;
        if (!left || r >= dealt) continue;
        int lo = 0, hi = n;                        // the last request that starts at r or before: the one that has it
        while (hi - lo > 1) {
            const int mid = (lo + hi) / 2;
            if (start[mid] <= r) lo = mid;
            else hi = mid;
        }
        int end = start[lo + 1];
        int64_t entry = (int64_t)seq_s[lo] * a.book.max_pages + have[lo] - start[lo];      // of its first page, less that one's rank
        for (; left && r < dealt; left &= left - 1, ++r) {
            if (r >= end) {
                while (start[lo + 1] <= r) ++lo;
                end = start[lo + 1];
                entry = (int64_t)seq_s[lo] * a.book.max_pages + have[lo] - start[lo];
            }
            a.book.table[entry + r] = 32 * w + __ffs((int)left) - 1;
        }
    }
}

// What is told of row `row`: token p of request i, in page id.
__device__ __forceinline__ void step_row(const StepArgs& a, int64_t row, int i, int p, int id) {
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
    if (a.out.slots) a.out.slots[row] = (int64_t)id * a.book.page_tokens + (p - step_whole(a, (uint32_t)p) * a.book.page_tokens);
}

constexpr int kWriteThreads = 256, kWriteItems = 1024, kWriteMost = 64;    // items of a workgroup, workgroups of a request

// Request blockIdx.x: entries of its row of the page table, the bits of its new pages, and its rows.
__global__ __launch_bounds__(kWriteThreads) void pages_write_kernel(StepArgs a) {
    const int i = blockIdx.x, len = a.out.kv_len[i], row0 = a.out.q_start[i], added = a.out.q_start[i + 1] - row0;
    const int seq = a.step.seq ? a.step.seq[i] : i, now = step_pages(a, len), have = step_pages(a, len - added);
    const int32_t* from = a.book.table + (int64_t)(now ? seq : 0) * a.book.max_pages;        // a refused one has no pages
    int32_t* to = a.out.page_table + i * a.out.table_stride;
    const int64_t x0 = (int64_t)blockIdx.y * kWriteThreads + threadIdx.x, step = (int64_t)gridDim.y * kWriteThreads;
    if (x0 == 0 && a.out.status[i] != VEDA_STEP_REFUSED) {
        if (a.step.grow[i] && !added) a.out.status[i] = VEDA_STEP_NO_ROOM;
        a.book.length[seq] = len;
    }
    for (int64_t x = x0; x < a.book.max_pages; x += step) {
        const int id = x < now ? from[x] : -1;
        if (x >= have && x < now) atomicOr(&a.book.used[id >> 5], 1u << (id & 31));
        to[x] = id;
    }
    for (int64_t r = x0; r < added; r += step) {
        const int p = len - added + (int)r;
        step_row(a, row0 + r, i, p, from[step_whole(a, (uint32_t)p)]);
    }
}

// All of it by one workgroup, for what fits: up to kOneRequests requests, kOneEntries entries of their rows of the table, kOneRows rows and kOneList
// pages dealt out at most, and what they take of LDS.
constexpr int kOneRequests = 1024, kOneEntries = 16384, kOneRows = 16384, kOneList = 4096;
inline size_t step_one_bytes(int64_t words, int64_t n, int64_t width, int64_t seqs) { return 4 * (size_t)(words + kOneList + std::max(n * width, seqs) + 5 * n + 1); }

// As many threads to a request, a power of two, as there are.
__global__ __launch_bounds__(kDealThreads) void pages_step_kernel(StepArgs a, int log_team) {
    extern __shared__ int one_smem[];
    __shared__ int part[3][kDealWaves];
    __shared__ int top_s[2];
    const int n = a.step.seqs, words = (a.book.pages + 31) / 32, width = a.book.max_pages, tid = threadIdx.x;
    const int i = tid >> log_team, team = 1 << log_team, t = tid & (team - 1);
    const bool mine = i < n, first = mine && t == 0;
    uint32_t* bits = reinterpret_cast<uint32_t*>(one_smem);          // [words]
    int* list = one_smem + words;                                    // [kOneList] pages dealt out
    int* page_s = list + kOneList;                                   // [n][width] the requests' rows of the table
    int* first_s = page_s;                                           // [max_seqs] before: the first request about a sequence
    int* have_s = page_s + max(n * width, a.book.max_seqs);          // of the requests, [n] each: pages kept
    int* kept_s = have_s + n;                                        // tokens kept
    int* open_s = kept_s + n;                                        // the page that the next token falls into
    int* start_s = open_s + n;                                       // pages dealt out before
    int* row_s = start_s + n;                                        // [n + 1] rows before
    const int seq = mine ? a.step.seq ? a.step.seq[i] : i : -1;
    const bool known = seq >= 0 && seq < a.book.max_seqs;
    for (int x = tid; x < a.book.max_seqs; x += kDealThreads) first_s[x] = n;
    for (int w = tid; w < words; w += kDealThreads) bits[w] = a.book.used[w];
    if (tid < 2) top_s[tid] = 0;
    __syncthreads();
    if (known && first) atomicMin(&first_s[seq], i);
    __syncthreads();
    StepAsk k{-1, 0, -1, -1, 0, 0, 0, 0};
    if (mine) k = step_ask(a, i, seq, known && first_s[seq] != i);
    __syncthreads();
    // What goes back; the others stay in page_s.  Four entries at a time.
    int32_t* row = a.book.table + (int64_t)max(k.kept < 0 ? 0 : k.seq, 0) * width;
    for (int j0 = t; mine && j0 < width; j0 += 4 * team) {
        int id[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int j = j0 + e * team;
            id[e] = j < min(k.cut_to, width) ? row[j] : -1;          // none of a refused one
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int j = j0 + e * team;
            if (j >= width) continue;
            const bool gone = id[e] != -1 && (j >= k.cut_from || (j >= k.evict_from && j < k.evict_to));
            if (gone) {
                if (id[e] >= 0 && id[e] < a.book.pages) atomicAnd(&bits[id[e] >> 5], ~(1u << (id[e] & 31)));   // bits go in any order
                row[j] = -1;
            }
            page_s[i * width + j] = gone ? -1 : id[e];
        }
    }
    __syncthreads();
    // Sums of free pages over the threads' words, and of pages and rows over the requests.  32 bits do: a request needs no more than `width` pages,
    // and rows count for one more than there are at most.
    const int each_w = (words + kDealThreads - 1) / kDealThreads, w0 = min(words, tid * each_w), w1 = min(words, w0 + each_w);
    const int need = k.kept < 0 ? 0 : step_pages(a, k.kept + k.grow) - k.cut_from, grow = k.kept < 0 ? 0 : min(k.grow, a.step.rows + 1);
    int sum[3] = {0, first ? need : 0, first ? grow : 0}, before[3], all[3];
    for (int w = w0; w < w1; ++w) sum[0] += __popc(step_free(a, w, bits[w]));
    sums_before(sum, part, before, all);
    // a request is served if the sums up to it fit, and so do all before it; the last one's sums are what is dealt out
    const int pages0 = first ? before[1] : before[1] - need, rows0 = first ? before[2] : before[2] - grow;      // before the request
    const bool fits = pages0 + need <= all[0] && rows0 + grow <= a.step.rows, fitted = pages0 <= all[0] && rows0 <= a.step.rows;
    last_of(&top_s[0], first && fits ? pages0 + need : 0);
    last_of(&top_s[1], first && fits ? rows0 + grow : 0);
    __syncthreads();
    const int dealt = top_s[0], rows = top_s[1], start = fitted ? pages0 : dealt;
    if (first) {
        const int len = k.kept < 0 ? 0 : k.kept + (fits ? k.grow : 0), at = fitted ? rows0 : rows;
        have_s[i] = k.cut_from;
        kept_s[i] = k.kept;
        open_s[i] = k.open;
        start_s[i] = start;
        row_s[i] = at;
        if (k.kept >= 0) a.book.length[k.seq] = len;
        a.out.q_start[i] = at;
        a.out.kv_len[i] = len;
        a.out.status[i] = k.kept < 0 ? VEDA_STEP_REFUSED : fits || k.grow == 0 ? VEDA_STEP_SERVED : VEDA_STEP_NO_ROOM;
    }
    if (tid == 0) {
        row_s[n] = rows;
        a.out.q_start[n] = rows;
    }
    for (int w = w0, rank = before[0]; w < w1; ++w) {
        uint32_t taken = 0;
        for (uint32_t left = step_free(a, w, bits[w]); left && rank < dealt; left &= left - 1, ++rank) {
            list[rank] = 32 * w + __ffs((int)left) - 1;
            taken |= left & (0u - left);
        }
        a.book.used[w] = bits[w] | taken;
    }
    __syncthreads();
    const int now = k.kept < 0 ? 0 : k.cut_from + (fits ? need : 0);
    int32_t* to = a.out.page_table + i * a.out.table_stride;
    for (int j = t; mine && j < width; j += team) {
        int id = -1;
        if (j < now) {
            id = page_s[i * width + j];
            if (j >= k.cut_from) row[j] = id = list[start + j - k.cut_from];
        }
        to[j] = id;
    }
    for (int r = tid; r < rows; r += kDealThreads) {
        int lo = 0, hi = n;                        // the last request that begins at r or before
        while (hi - lo > 1) {
            const int mid = (lo + hi) / 2;
            if (row_s[mid] <= r) lo = mid;
            else hi = mid;
        }
        const int p = kept_s[lo] + r - row_s[lo], x = step_whole(a, (uint32_t)p);
        step_row(a, r, lo, p, x < have_s[lo] ? open_s[lo] : list[start_s[lo] + x - have_s[lo]]);
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
        for (const int32_t* res : {out->page_table, out->kv_len, out->q_start, out->status, out->positions, out->row_seq, book->table, book->length, (int32_t*)book->used})
            if (in && (in == res || in == (const int32_t*)out->slots)) return VEDA_ERR_INVALID_ARG;
    if (book->pages > 1 << 19 || book->max_seqs > 8192 || step->seqs > 8192 || step->rows > 1 << 30) return VEDA_ERR_UNSUPPORTED;
    if ((int64_t)book->max_pages * book->page_tokens > (int64_t)1 << 30) return VEDA_ERR_UNSUPPORTED;
    const hipStream_t s = (hipStream_t)stream;
    int shift = 31;
    while ((uint64_t)1 << (shift - 31) < (uint64_t)book->page_tokens) ++shift;
    const veda::StepArgs a{*book, *step, *out, (uint32_t)((((uint64_t)1 << shift) + book->page_tokens - 1) / book->page_tokens), shift};
    const int64_t n = step->seqs, words = (book->pages + 31) / 32, grows = std::min(step->max_new, step->rows);
    veda_status st = VEDA_OK;
    // One kernel as long as one compute unit writes it all as fast as the launches of three take.
    if (n > 0 && n <= veda::kOneRequests && n * book->max_pages <= veda::kOneEntries && std::min<int64_t>(n * grows, step->rows) <= veda::kOneRows &&
        n * (grows / book->page_tokens + 1) <= veda::kOneList && veda::step_one_bytes(words, n, book->max_pages, book->max_seqs) <= (size_t)veda::kStepLds) {
        const size_t lds = veda::step_one_bytes(words, n, book->max_pages, book->max_seqs);
        if (lds > 64 * 1024) VEDA_HIP_TRY(hipFuncSetAttribute((const void*)veda::pages_step_kernel, hipFuncAttributeMaxDynamicSharedMemorySize, veda::kStepLds));
        int log_team = 0;
        while (n << (log_team + 1) <= veda::kDealThreads) ++log_team;
        hipLaunchKernelGGL(veda::pages_step_kernel, dim3(1), dim3(veda::kDealThreads), lds, s, a, log_team);
        return veda::launch_status("veda_pages_step");
    }
    if (n) {
        hipLaunchKernelGGL(veda::pages_give_back_kernel, dim3((unsigned)n), dim3(veda::kGiveThreads), 0, s, a);
        st = veda::launch_status("veda_pages_step");
        if (st != VEDA_OK) return st;
    }
    const size_t lds = 4 * ((size_t)words + 2 * (size_t)n + 1) + 2 * (size_t)n;
    if (lds > 64 * 1024) VEDA_HIP_TRY(hipFuncSetAttribute((const void*)veda::pages_deal_kernel, hipFuncAttributeMaxDynamicSharedMemorySize, veda::kStepLds));
    const int64_t most = n * (grows / book->page_tokens + 1);       // pages dealt out
    hipLaunchKernelGGL(veda::pages_deal_kernel, dim3((unsigned)std::max<int64_t>(1, std::min<int64_t>(16, most / 1024))), dim3(veda::kDealThreads), lds, s, a);
    st = veda::launch_status("veda_pages_step");
    if (st != VEDA_OK || !n) return st;
    const int64_t widest = std::max<int64_t>(book->max_pages, grows);
    hipLaunchKernelGGL(veda::pages_write_kernel, dim3((unsigned)n, (unsigned)std::min<int64_t>(veda::kWriteMost, (widest + veda::kWriteItems - 1) / veda::kWriteItems)),
                       dim3(veda::kWriteThreads), 0, s, a);
    return veda::launch_status("veda_pages_step");
}
