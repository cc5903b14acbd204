// Checks that the entry points with strided [batch, heads, tokens, head_dim] tensors
// share (host code).
#pragma once

#include <utility>

#include "mosaic_bsa.h"

namespace bsa {

// Strides with the contiguous case written out.
inline mosaic_bsa_strides strides_of(const mosaic_bsa_strides& s, int64_t heads, int64_t tokens,
                                     int64_t D)
{
    if (s.token != 0) return s;
    return mosaic_bsa_strides{heads * tokens * D, tokens * D, D};
}

// Strides that no [batch, heads, tokens, D] tensor has: negative, more than 2^40 elements, or, in an
// output, too short for a row.
inline bool bad_strides(const mosaic_bsa_strides& s, int64_t batch, int64_t heads, int64_t tokens,
                        int64_t D, bool output)
{
    if (s.token == 0) return false;                    // contiguous
    const int64_t most = (int64_t)1 << 40;
    if (s.batch < 0 || s.head < 0 || s.token < 0 || s.batch > most || s.head > most ||
        s.token > most)
        return true;
    if (!output) return false;
    return (batch > 1 && s.batch < D) || (heads > 1 && s.head < D) || (tokens > 1 && s.token < D);
}

// Whether rows of an output may share memory: from the smallest stride on, each has to step over all
// that the dimensions before it reach.
inline bool rows_meet(const mosaic_bsa_strides& s, int64_t batch, int64_t heads, int64_t tokens, int64_t D)
{
    if (s.token == 0) return false;
    struct { int64_t stride, n; } d[3] = {{s.batch, batch}, {s.head, heads}, {s.token, tokens}};
    const auto order = [&](int i, int j) {
        if (d[j].stride < d[i].stride) std::swap(d[i], d[j]);
    };
    order(0, 1);
    order(1, 2);
    order(0, 1);
    int64_t reach = D;
    for (const auto& x : d) {
        if (x.n <= 1) continue;
        if (x.stride < reach || x.n > ((int64_t)1 << 60) / x.stride) return true;
        reach += x.stride * (x.n - 1);
    }
    return false;
}

}  // namespace bsa
