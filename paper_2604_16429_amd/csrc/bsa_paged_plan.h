// Attention over a cache in pages: which tokens a query sees and where they lie.  Plain arithmetic, for
// host and device.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "mosaic_bsa.h"

namespace bsa {

namespace paged {

constexpr int32_t kUnbounded = 1 << 30;

struct Shape {
    int32_t batch, heads, kv_heads, group;
    int32_t q_tokens, rows;                // rows = q_tokens * group
    int32_t pages, page_shift, table_pages, prefix_tokens;
    int32_t left, sinks;                   // left: kUnbounded = no bound
    float scale;
    const int32_t *q_lens, *k_lens, *table, *prefix_table, *prefix_len;    // q_lens, prefix_len: or null
    mosaic_bsa_strides q, out, k, v;       // elements; k, v: `batch` steps from page to page
};

// Lengths of a sequence, held to what the tensors have.
struct Sequence {
    int ql, kl, prefix;
};

// The tokens that queries at places first .. last see, in tiles of KT: tiles of the prefix, then of the
// sequence's own tokens, each from its beginning (so that pages and tiles start together), sinks
// first.  `skip` tiles of a part lie between its sinks and what the window reaches.
struct Part {
    int sinks, count, skip;                // in tiles
    __host__ __device__ inline int tile(int t) const { return t < sinks ? t : t + skip; }
};
template <int KT>
__host__ __device__ inline Part part_of(int tokens, int lo, int hi, int sinks)
{
    // places lo .. hi and below `sinks`, counted from the part's beginning; it has `tokens`
    Part p;
    const int end = (max(0, min(tokens, hi + 1)) + KT - 1) / KT;
    p.sinks = min((max(0, min(sinks, tokens)) + KT - 1) / KT, end);
    const int from = max(p.sinks, min(max(lo, 0) / KT, end));
    p.skip = from - p.sinks;
    p.count = p.sinks + end - from;
    return p;
}
struct Tile {
    int at, count;                         // index of its first token in the part; tokens of the part
    int token;                             // the first token's place in the sequence
    bool shared;
};
template <int KT>
struct Tiles {
    Part shared, own;
    int prefix, kl, count;
    __host__ __device__ inline Tiles(const Shape& s, const Sequence& q, int first, int last)
    {
        const int lo = first - s.left;     // (left is at most 2^30, places are below it)
        prefix = q.prefix;
        kl = q.kl;
        shared = part_of<KT>(q.prefix, lo, last, s.sinks);
        own = part_of<KT>(q.kl, lo - q.prefix, last - q.prefix, s.sinks - q.prefix);
        count = shared.count + own.count;
    }
    __host__ __device__ inline Tile operator[](int t) const
    {
        Tile x;
        x.shared = t < shared.count;
        x.at = (x.shared ? shared.tile(t) : own.tile(t - shared.count)) * KT;
        x.count = x.shared ? prefix : kl;
        x.token = x.shared ? x.at : prefix + x.at;
        return x;
    }
};

// The page that holds token `at` of a part, or -1.
__host__ __device__ inline int page_of(const Shape& s, const int32_t* table, int at, int count)
{
    if (at >= count) return -1;
    const int id = table[at >> s.page_shift];
    return (uint32_t)id < (uint32_t)s.pages ? id : -1;
}

}  // namespace paged

}  // namespace bsa
