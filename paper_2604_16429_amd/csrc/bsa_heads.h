// Checks that the entry points with strided [batch, heads, tokens, head_dim] tensors
// share (host code).
#pragma once

#include "mosaic_bsa.h"

namespace bsa {

// Strides with the contiguous case written out.
inline mosaic_bsa_strides strides_of(const mosaic_bsa_strides& s, int64_t heads, int64_t tokens,
                                     int64_t D)
{
    if (s.token != 0) return s;
    return mosaic_bsa_strides{heads * tokens * D, tokens * D, D};
}

// Strides that a [batch, heads, tokens, D] tensor may have: 2^40 elements at most, and in an
// output no two rows at one place.
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

}  // namespace bsa
