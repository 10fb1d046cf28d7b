// Pages of a paged cache: who holds which.  Host arithmetic without HIP types.  Not part of the public ABI.
#pragma once

#include <stdint.h>

#include <algorithm>
#include <functional>
#include <queue>
#include <vector>

namespace veda {

// The invariant: holders[p] = number of table entries that name page p; a page is in `free` exactly when that is 0.
class PageBook {
  public:
    enum Result { kOk, kBadArg, kNoRoom };

    PageBook(int32_t pages, int32_t page_tokens, int32_t max_seqs, int32_t max_pages)
        : page_tokens_(page_tokens), max_pages_(max_pages), holders_((size_t)pages, 0), length_((size_t)max_seqs, 0),
          table_((size_t)max_seqs * max_pages, -1) {
        std::vector<int32_t> all((size_t)pages);
        for (int32_t p = 0; p < pages; ++p) all[(size_t)p] = p;
        free_ = Free(std::greater<int32_t>(), std::move(all));
    }

    const int32_t* table() const { return table_.data(); }
    bool has(int32_t seq) const { return seq >= 0 && (size_t)seq < length_.size(); }
    int32_t length(int32_t seq) const { return length_[(size_t)seq]; }
    int32_t free_count() const { return (int32_t)free_.size(); }

    Result extend(int32_t seq, int32_t tokens, int32_t* copies, int32_t capacity, int32_t* n_copies) {
        if (!has(seq) || tokens < length(seq) || capacity < 0 || pages_of(tokens) > max_pages_) return kBadArg;
        int32_t* row = row_of(seq);
        const int32_t old = length(seq), have = pages_of(old), want = pages_of(tokens);
        // the page that the next token falls into, if it has tokens already
        const bool open = tokens > old && old % page_tokens_ != 0;
        const int32_t last = open ? row[have - 1] : -1;
        const bool own = last >= 0 && holders_[(size_t)last] > 1;     // shared: a page of its own, copied
        if (open && last < 0) return kBadArg;                         // evicted, then cut open: its first tokens are gone
        if (want - have + own > free_count() || (own && (capacity < 1 || !copies))) return kNoRoom;
        if (own) {
            const int32_t p = take();
            copies[0] = last;
            copies[1] = p;
            --holders_[(size_t)last];
            row[have - 1] = p;
        }
        for (int32_t i = have; i < want; ++i) row[i] = take();
        length_[(size_t)seq] = tokens;
        *n_copies = own;
        return kOk;
    }

    Result fork(int32_t from, int32_t to) {
        if (!has(from) || !has(to) || from == to || length(to) != 0) return kBadArg;
        for (int32_t i = 0; i < pages_of(length(from)); ++i) {
            row_of(to)[i] = row_of(from)[i];
            if (row_of(to)[i] >= 0) ++holders_[(size_t)row_of(to)[i]];
        }
        length_[(size_t)to] = length(from);
        return kOk;
    }

    Result truncate(int32_t seq, int32_t tokens) {
        if (!has(seq) || tokens < 0 || tokens > length(seq)) return kBadArg;
        for (int32_t i = pages_of(tokens); i < pages_of(length(seq)); ++i) drop(row_of(seq)[i]);
        length_[(size_t)seq] = tokens;
        return kOk;
    }

    Result evict(int32_t seq, int32_t first, int32_t last) {
        if (!has(seq) || first < 0 || last < first || last > length(seq)) return kBadArg;
        for (int32_t i = pages_of(first); i < last / page_tokens_; ++i) drop(row_of(seq)[i]);
        return kOk;
    }

    // Pages in use above their number move, highest first, into the lowest free ones: sources and targets are disjoint.
    Result compact(int32_t* copies, int32_t capacity, int32_t* n_copies) {
        if (capacity < 0) return kBadArg;
        const int32_t pages = (int32_t)holders_.size(), used = pages - free_count();
        std::vector<int32_t> to;            // page -> where it goes
        int32_t moves = 0;
        for (int32_t p = used; p < pages; ++p) moves += holders_[(size_t)p] > 0;
        if (moves > capacity || (moves && !copies)) return kNoRoom;
        if (moves) {
            to.resize((size_t)pages);
            std::vector<int32_t> left;      // free pages afterwards: all from `used` on
            left.reserve((size_t)pages);         // drop never allocates
            for (int32_t p = used; p < pages; ++p) left.push_back(p);
            Free after(std::greater<int32_t>(), std::move(left));   // the last allocation: from here on nothing fails
            int32_t hole = 0;
            moves = 0;
            for (int32_t p = pages - 1; p >= used; --p) {
                if (!holders_[(size_t)p]) continue;
                while (holders_[(size_t)hole]) ++hole;
                copies[2 * moves] = p;
                copies[2 * moves + 1] = hole;
                ++moves;
                to[(size_t)p] = hole;
                holders_[(size_t)hole] = holders_[(size_t)p];
                holders_[(size_t)p] = 0;
            }
            for (int32_t& e : table_)
                if (e >= used) e = to[(size_t)e];
            free_.swap(after);
        }
        *n_copies = moves;
        return kOk;
    }

  private:
    typedef std::priority_queue<int32_t, std::vector<int32_t>, std::greater<int32_t>> Free;

    int32_t pages_of(int32_t tokens) const { return (int32_t)(((int64_t)tokens + page_tokens_ - 1) / page_tokens_); }
    int32_t* row_of(int32_t seq) { return table_.data() + (size_t)seq * (size_t)max_pages_; }
    int32_t take() {
        const int32_t p = free_.top();
        free_.pop();
        holders_[(size_t)p] = 1;
        return p;
    }
    // free_ always has room for every page, so the push cannot fail.
    void drop(int32_t& entry) {
        if (entry < 0) return;
        if (--holders_[(size_t)entry] == 0) free_.push(entry);
        entry = -1;
    }

    int32_t page_tokens_, max_pages_;
    std::vector<int32_t> holders_, length_, table_;
    Free free_;
};

}  // namespace veda
