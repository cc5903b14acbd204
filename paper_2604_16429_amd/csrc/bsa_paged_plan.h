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
// Which of a sequence's tokens a list holds.
enum Which { kAll, kShared, kOwn };
template <int KT>
struct Tiles {
    Part shared, own;
    int prefix, kl, count;
    __host__ __device__ inline Tiles(const Shape& s, const Sequence& q, int first, int last, Which which = kAll)
    {
        const int lo = first - s.left;     // (left is at most 2^30, places are below it)
        prefix = q.prefix;
        kl = q.kl;
        shared = own = Part{0, 0, 0};
        if (first <= last) {
            if (which != kOwn) shared = part_of<KT>(q.prefix, lo, last, s.sinks);
            if (which != kShared)
                own = part_of<KT>(q.kl, lo - q.prefix, last - q.prefix, s.sinks - q.prefix);
        }
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

// How a call is dealt out.  Tokens of few rows are split over workgroups, whose sums a second launch joins.
//
// The prefix's part of rows that are too few to fill a tile by themselves is worked on for the rows of all
// sequences together ("stacked"), in `shared_splits` shares of its tokens; without that the prefix
// is the beginning of every sequence.  What is left of a sequence, u units of 128 tokens, is cut into
// max(1, ceil(u / c)) chunks (stacked: maybe none), c the same for all and large enough that there are
// at most `chunks` of them, and at least `least`: with U the sum of all u, c = max(least, ceil(U / (chunks -
// batch))).  Lengths are in device memory: workgroups find their chunk by a sum over the batch.
constexpr int kUnit = 128;
constexpr int kMostScanned = 1024;         // sequences; a larger batch has a chunk for each
struct Plan {
    bool stacked, parts;                   // parts: there may be several sums of one row
    bool scanned;                          // chunks are looked up; else chunk i is sequence i
    int32_t chunks, least, shared_splits;
    int32_t all_rows;                      // batch x rows
    float* acc;                            // sums of weight x value against a reference: [kv_heads][chunks][rows][D],
    float2* ml;                            // then [kv_heads][shared_splits][all_rows][D]; (reference in base 2, sum
                                           // of weights) likewise
    // index of a row's sums
    __host__ __device__ inline int64_t own_part(const Shape& s, int a, int chunk, int row) const
    {
        return ((int64_t)a * chunks + chunk) * s.rows + row;
    }
    __host__ __device__ inline int64_t shared_part(const Shape& s, int a, int split, int row) const
    {
        return (int64_t)s.kv_heads * chunks * s.rows +
               ((int64_t)a * shared_splits + split) * all_rows + row;
    }
    __host__ __device__ inline int64_t all_parts(const Shape& s) const
    {
        return (int64_t)s.kv_heads * ((int64_t)chunks * s.rows + (int64_t)shared_splits * all_rows);
    }
};
// Units of a sequence and the chunks that they make.
__host__ __device__ inline int units_of(const Shape& s, const Plan& plan, const Sequence& q)
{
    const int p0 = q.prefix + q.kl - q.ql;
    const Tiles<32> tiles(s, q, p0, p0 + q.ql - 1, plan.stacked ? kOwn : kAll);
    return (tiles.count + kUnit / 32 - 1) / (kUnit / 32);
}
__host__ __device__ inline int chunk_units(const Shape& s, const Plan& plan, int all_units)
{
    const int room = plan.chunks - s.batch, c = (all_units + room - 1) / room;
    return c > plan.least ? c : plan.least;
}
__host__ __device__ inline int chunks_of(const Plan& plan, int units, int per_chunk)
{
    const int n = (units + per_chunk - 1) / per_chunk;
    return n > 0 || plan.stacked ? n : 1;
}

// Rows of a workgroup's tile, by how many there are.
inline int tile_rows(int64_t rows) { return rows <= 16 ? 16 : 32; }
// Most tokens that a sequence's list can hold.
inline int64_t most_tokens(const Shape& s, bool stacked)
{
    const int64_t own = (int64_t)s.table_pages << s.page_shift, all = own + (stacked ? 0 : s.prefix_tokens);
    const int64_t seen = (int64_t)s.left + s.q_tokens + s.sinks;
    return seen < all ? seen : all;
}
// Nothing here may depend on strides, which the size of the workspace is asked for without.
inline Plan make_plan(const Shape& s)
{
    Plan p = {};
    p.all_rows = 1;
    const int64_t own = (int64_t)s.table_pages << s.page_shift;
    p.stacked = s.batch > 1 && s.prefix_tokens >= 256 && s.rows < 128 && s.left >= s.prefix_tokens + own;
    if (p.stacked) {
        p.all_rows = s.batch * s.rows;
        const int tile = tile_rows(p.all_rows);
        const int64_t items = (int64_t)s.kv_heads * ((p.all_rows + tile - 1) / tile);
        int64_t n = 512 / items;
        if (n > s.prefix_tokens / 256) n = s.prefix_tokens / 256;
        p.shared_splits = n < 1 ? 1 : n >= 8 ? (int)n & ~7 : (int)n;
    }
    const int64_t tokens = most_tokens(s, p.stacked), units = (tokens + 31) / 32 / (kUnit / 32) + 2;
    const int tile = tile_rows(s.rows);
    const int64_t tiles = (int64_t)s.kv_heads * ((s.rows + tile - 1) / tile);
    p.least = 2;
    int64_t n = 1024 / tiles;
    if (n < 2 * (int64_t)s.batch) n = 2 * (int64_t)s.batch;
    const int64_t most = s.batch * ((units + p.least - 1) / p.least);
    if (n > most) n = most;
    if (s.batch > kMostScanned || s.batch * units >= 1 << 30 || s.batch * tiles >= 4096 || tokens < 640)
        n = s.batch;
    p.scanned = n > s.batch;
    p.chunks = (int)n;
    p.parts = p.stacked || p.scanned;
    return p;
}

// The page that holds token `at` of a part, or -1.
__host__ __device__ inline int page_of(const Shape& s, const int32_t* table, int at, int count)
{
    if (at >= count) return -1;
    const int id = table[at >> s.page_shift];
    return (uint32_t)id < (uint32_t)s.pages ? id : -1;
}

}  // namespace paged

}  // namespace bsa
