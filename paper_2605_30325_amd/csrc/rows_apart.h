// Whether the rows that a call writes are rows of their own.  Host arithmetic without HIP types.  Not part of the public ABI.
#pragma once

#include <stdint.h>

#include <algorithm>

namespace veda {

struct RowAxis { int64_t count, stride; };   // elements; stride >= 0
enum class RowsApart { kApart, kShare, kTooMany };

// Rows of d elements, one for every combination of the axes' indexes: does any element belong to two of them?  Where every stride covers all
// that the smaller ones reach, as in any slice of a dense tensor, it does not.  Other strides may still keep rows apart (2 x 3 rows of 128 at
// 384 and 256): for every difference of two indexes the third one's that comes nearest is looked at, up to 2^22 differences.
inline RowsApart rows_apart(RowAxis a, RowAxis b, RowAxis c, int64_t d) {
    typedef __int128 Wide;
    RowAxis x[3] = {a, b, c};
    for (RowAxis& e : x)
        if (e.count < 2) e = RowAxis{1, 0};
    std::sort(x, x + 3, [](const RowAxis& p, const RowAxis& q) { return p.stride < q.stride; });
    Wide reach = d;
    bool within = true;
    for (const RowAxis& e : x) {
        if (e.count < 2) continue;
        if (e.stride < d) return RowsApart::kShare;
        within = within && e.stride >= reach;
        reach += (Wide)(e.count - 1) * e.stride;
    }
    if (within) return RowsApart::kApart;
    std::sort(x, x + 3, [](const RowAxis& p, const RowAxis& q) { return p.count < q.count; });
    if ((Wide)x[0].count * (2 * (Wide)x[1].count - 1) > 1 << 22) return RowsApart::kTooMany;
    for (int64_t i = 0; i < x[0].count; ++i)
        for (int64_t j = 1 - x[1].count; j < x[1].count; ++j) {
            const Wide at = (Wide)i * x[0].stride + (Wide)j * x[1].stride, far = at < 0 ? -at : at;
            const Wide low = std::min<Wide>(far / x[2].stride, x[2].count - 1);
            for (Wide k = low; k <= low + 1 && k < x[2].count; ++k) {
                const Wide gap = far - k * x[2].stride;
                if ((i || j || k) && gap < d && -gap < d) return RowsApart::kShare;
            }
        }
    return RowsApart::kApart;
}

}  // namespace veda
