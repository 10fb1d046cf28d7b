// The page book behind its C entry points: checks, and no exception leaves a call.
#include <new>

#include "pages.h"
#include "veda_internal.h"

struct veda_pages {
    veda::PageBook book;
};

static veda_status told(veda::PageBook::Result r, const char* what) {
    if (r == veda::PageBook::kBadArg) return VEDA_ERR_INVALID_ARG;
    if (r == veda::PageBook::kNoRoom) {
        veda::set_last_error(std::string(what) + ": not enough free pages, or no room for the copies");
        return VEDA_ERR_WORKSPACE;
    }
    return VEDA_OK;
}

extern "C" {

veda_status veda_pages_create(int32_t pages, int32_t page_tokens, int32_t max_seqs, int32_t max_pages, veda_pages** out) {
    if (!out || pages < 1 || page_tokens < 1 || max_seqs < 1 || max_pages < 1) return VEDA_ERR_INVALID_ARG;
    if ((int64_t)max_pages * page_tokens > (int64_t)1 << 30 || (int64_t)max_seqs * max_pages > (int64_t)1 << 31) return VEDA_ERR_UNSUPPORTED;
    try {
        *out = new veda_pages{veda::PageBook(pages, page_tokens, max_seqs, max_pages)};
        return VEDA_OK;
    } catch (const std::exception&) {
        return veda::hip_fail(hipErrorOutOfMemory, "veda_pages_create");
    }
}

void veda_pages_destroy(veda_pages* p) { delete p; }

const int32_t* veda_pages_table(const veda_pages* p) { return p ? p->book.table() : nullptr; }

int32_t veda_pages_length(const veda_pages* p, int32_t seq) { return p && p->book.has(seq) ? p->book.length(seq) : -1; }

int32_t veda_pages_free_count(const veda_pages* p) { return p ? p->book.free_count() : -1; }

veda_status veda_pages_extend(veda_pages* p, int32_t seq, int32_t tokens, int32_t* copies, int32_t capacity, int32_t* n_copies) {
    if (!p || !n_copies) return VEDA_ERR_INVALID_ARG;
    return told(p->book.extend(seq, tokens, copies, capacity, n_copies), "veda_pages_extend");
}

veda_status veda_pages_fork(veda_pages* p, int32_t from, int32_t to) {
    return p ? told(p->book.fork(from, to), "veda_pages_fork") : VEDA_ERR_INVALID_ARG;
}

veda_status veda_pages_truncate(veda_pages* p, int32_t seq, int32_t tokens) {
    return p ? told(p->book.truncate(seq, tokens), "veda_pages_truncate") : VEDA_ERR_INVALID_ARG;
}

veda_status veda_pages_evict(veda_pages* p, int32_t seq, int32_t first, int32_t last) {
    return p ? told(p->book.evict(seq, first, last), "veda_pages_evict") : VEDA_ERR_INVALID_ARG;
}

veda_status veda_pages_compact(veda_pages* p, int32_t* copies, int32_t capacity, int32_t* n_copies) {
    if (!p || !n_copies) return VEDA_ERR_INVALID_ARG;
    try {
        return told(p->book.compact(copies, capacity, n_copies), "veda_pages_compact");
    } catch (const std::exception&) {
        return veda::hip_fail(hipErrorOutOfMemory, "veda_pages_compact");
    }
}

}  // extern "C"
