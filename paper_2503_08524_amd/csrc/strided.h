// Rows in memory by three strides: whether outputs lie on each other.
#pragma once
#include <algorithm>
#include <cstdint>

namespace d3 {

struct Strided { int64_t n, stride; };     // a dim: entries, elements from one to the next

// Rows of `width` elements at sum i_j stride_j, 0 <= i_j < n_j, and the same `apart` elements on (0: there is one such set only).  False: no two of these rows have an element in common.  The dims have to be nested: in
// the order of their strides each passes over all that those before it span (rows that interleave in another way are taken as overlapping, though some are not).
inline bool rows_overlap(int64_t width, const Strided (&dims)[3], __int128 apart) {
    Strided d[3];
    int n = 0;
    for (const Strided& x : dims) if (x.n > 1) d[n++] = {x.n, x.stride};
    auto size = [](int64_t s) { return s < 0 ? -(__int128)s : (__int128)s; };
    std::sort(d, d + n, [&](const Strided& a, const Strided& b) { return size(a.stride) < size(b.stride); });
    __int128 span = width;
    for (int j = 0; j < n; ++j) {
        if (size(d[j].stride) < span) return true;
        span += (d[j].n - 1) * size(d[j].stride);
    }
    if (apart == 0) return false;
    // The two sets meet where some differences of indexes bring `apart` below a row's width.  What the smaller dims can add is less than a stride, so of every dim only the two multiples around what is left count.
    struct Search {
        static bool from(const Strided* d, int n, __int128 left, int64_t width) {
            if (n == 0) return left < width && -left < width;
            const __int128 s = d[n - 1].stride < 0 ? -(__int128)d[n - 1].stride : (__int128)d[n - 1].stride;
            const __int128 below = left >= 0 ? left / s : -((-left + s - 1) / s);
            for (__int128 i = below; i <= below + 1; ++i)
                if (i < d[n - 1].n && -i < d[n - 1].n && from(d, n - 1, left - i * s, width)) return true;
            return false;
        }
    };
    return Search::from(d, n, apart, width);
}

}  // namespace d3
