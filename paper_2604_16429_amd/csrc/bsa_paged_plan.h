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

// How a call is dealt out.  Workgroups own tiles of a sequence's rows ("entries", all sequences' last tiles
// first: they see most) and walk the tokens that these see; few rows see many tokens, which are then
// split over workgroups, whose sums a second launch joins.
//
// The prefix's part of rows that are too few to fill a tile by themselves is worked on for the rows of all
// sequences together ("stacked"), in `shared_splits` shares of its tokens; without that the prefix
// is the beginning of every sequence.  What is left of an entry, u units of 128 tokens, is cut into
// max(1, ceil(u / c)) chunks (stacked: maybe none), c the same for all and large enough that there are
// at most `chunks` of them.  Lengths are in device memory: workgroups find c and their chunk by sums over
// the entries.
constexpr int kUnit = 128, kLeast = 2;     // c is kLeast at least
constexpr int kMostScanned = 256;          // entries; more have a chunk each (400 sequences of up to 2,000, 2 heads:
                                           // 106 us, looked up 118; 130 of up to 4,000, 4 heads: 88, looked up 77).  That
                                           // costs long ones: 256 of up to 4,000, one head, 69 us, 257 83; up to 16,000 233, 360
struct Entry {
    int32_t first, chunks;
};
struct Plan {
    bool stacked, parts;                   // parts: there may be several sums of one row
    bool scanned;                          // chunks are looked up; else chunk i is entry i
    int32_t waves;                         // of a workgroup
    int32_t tile, tile_rows;               // rows of a workgroup at most, and those that there are
    int32_t row_tiles, entries, chunks;
    int32_t shared_tile, shared_splits, all_rows;      // all_rows = batch x rows
    float* acc;                            // sums of weight x value against a reference: [kv_heads][chunks][tile_rows][D],
    float2* ml;                            // then [kv_heads][shared_splits][all_rows][D]; (reference in base 2, sum
                                           // of weights) likewise
    Entry* found;                          // [entries]: what the first launch found, for the second
    // index of the sums of a chunk's first row
    __host__ __device__ inline int64_t own_part(int a, int chunk) const
    {
        return ((int64_t)a * chunks + chunk) * tile_rows;
    }
    __host__ __device__ inline int64_t shared_part(const Shape& s, int a, int split, int row) const
    {
        return (int64_t)s.kv_heads * chunks * tile_rows + ((int64_t)a * shared_splits + split) * all_rows + row;
    }
    __host__ __device__ inline int64_t all_parts(const Shape& s) const
    {
        return (int64_t)s.kv_heads * ((int64_t)chunks * tile_rows + (int64_t)shared_splits * all_rows);
    }
    __host__ __device__ inline int sequence_of(const Shape& s, int entry) const { return entry % s.batch; }
    __host__ __device__ inline int tile_of(const Shape& s, int entry) const { return row_tiles - 1 - entry / s.batch; }
    __host__ __device__ inline int entry_of(const Shape& s, int b, int tile_at) const
    {
        return (row_tiles - 1 - tile_at) * s.batch + b;
    }
};
// The tokens that an entry's chunks hold.
template <int KT>
__host__ __device__ inline Tiles<KT> tiles_of(const Shape& s, const Plan& plan, const Sequence& q, int tile_at)
{
    const int row0 = tile_at * plan.tile, end = row0 + plan.tile < s.rows ? row0 + plan.tile : s.rows;
    const int last = (end - 1) / s.group < q.ql - 1 ? (end - 1) / s.group : q.ql - 1;
    const int p0 = q.prefix + q.kl - q.ql;
    return Tiles<KT>(s, q, p0 + row0 / s.group, p0 + last, plan.stacked ? kOwn : kAll);
}
__host__ __device__ inline int units_of(const Shape& s, const Plan& plan, const Sequence& q, int tile_at)
{
    return (tiles_of<32>(s, plan, q, tile_at).count + kUnit / 32 - 1) / (kUnit / 32);
}
__host__ __device__ inline int chunks_of(const Plan& plan, int units, int per_chunk)
{
    const int n = (int)((uint32_t)(units + per_chunk - 1) / (uint32_t)per_chunk);
    return n > 0 || plan.stacked ? n : 1;
}
// The least c for which `all` units make no more chunks than there is room for: total(c) of them.
template <class Total>
__host__ __device__ inline int chunk_units(const Plan& plan, int all, Total total)
{
    const int room = plan.chunks - plan.entries;       // (each entry's last chunk may be short)
    int lo = (all + plan.chunks - 1) / plan.chunks, hi = (all + room - 1) / room;
    lo = lo > kLeast ? lo : kLeast;
    hi = hi > kLeast ? hi : kLeast;
    while (lo < hi) {
        const int mid = (lo + hi) / 2;
        if (total(mid) <= plan.chunks) hi = mid;
        else lo = mid + 1;
    }
    return hi;
}

// What decides beside the shape: the largest tiles of a sequence's rows and of those of all, how many wavefronts a
// workgroup has that takes all of up to `few` tokens of up to 16 rows, and the bytes of a key and a value.
struct Kind {
    int most_own, most_shared;
    int waves, few;
    int token_bytes;
};
// Rows of a workgroup's tile, by how many there are.
inline int tile_rows_of(int64_t rows, int most) { return rows <= 16 ? 16 : rows <= 32 ? 32 : most; }
// Most tokens that a sequence's list can hold.
inline int64_t most_tokens(const Shape& s, bool stacked)
{
    const int64_t own = (int64_t)s.table_pages << s.page_shift, all = own + (stacked ? 0 : s.prefix_tokens);
    const int64_t seen = (int64_t)s.left + s.q_tokens + s.sinks;
    return seen < all ? seen : all;
}
// Nothing here may depend on strides, which the size of the workspace is asked for without.
inline Plan make_plan(const Shape& s, int D, const Kind& kind)
{
    Plan p = {};
    p.waves = 4;
    p.tile = tile_rows_of(s.rows, kind.most_own);
    p.tile_rows = p.tile < s.rows ? p.tile : s.rows;
    p.row_tiles = (s.rows + p.tile - 1) / p.tile;
    p.entries = p.chunks = s.batch * p.row_tiles;
    p.all_rows = 1;
    const int64_t own = (int64_t)s.table_pages << s.page_shift;
    // The prefix is worked on for all together where that saves 24 MB of reads and more, mostly from L2: less does
    // not pay for joining.  us, apart | together: 16 rows of all, head dim 128, 4 sequences on 2,000 (12 MB) 12.6 |
    // 15.0, on 8,000 (49 MB) 21 | 15; head dim 64, 16 on 2,000 (30 MB) 16.7 | 16.7, on 8,000 25 | 15; fp32, 6 on 1,501 (4 MB)
    // 12.0 | 14.6; 24 members on 28,800 72 | 29.
    const int64_t saved = (int64_t)(s.batch - 1) * s.prefix_tokens * s.kv_heads * kind.token_bytes;
    // And where a sequence's reads of it are 12 times what one sum of each of its rows takes, out and in again, of which
    // there are two at least, a share's and a chunk's.  us, bf16, apart | together.  Left apart: head dim 128, 128 sequences of
    // 120 rows on 614 36 | 73, 1,003 on 777 143 | 286, 105 of 60 on 989 67 | 50; head dim 64, 288 of 96 on 1,966 53 | 44.
    // Together: head dim 128, 448 of 20 on 639 26 | 33, 897 of 120 on 3,710 240 | 298; fp32, head dim 128, 531 of 64 on 1,916
    // 2,582 | 1,723.  Of 820 drawn calls 82 took a quarter longer than the other way without this, 22 with it.
    const bool long_enough = (int64_t)s.prefix_tokens * kind.token_bytes >= (int64_t)12 * 2 * 4 * D * s.rows;
    p.stacked = s.prefix_tokens >= 256 && saved >= 24000000 && long_enough && s.rows < 128 &&
                s.left >= s.prefix_tokens + own;
    // (few rows and tokens: one launch)
    if (!p.stacked && s.rows <= 16 && kind.waves > 4 && most_tokens(s, false) <= kind.few) {
        p.waves = kind.waves;
        return p;
    }
    // Tiles of 128 rows: chunks and shares are as many as the chip holds in bf16 at head dims 64 and 128, shares of at
    // least 256 tokens, 384 where a share's sums are those of 128 rows.  us: 24 members on 28,800, shares of 256 39, 384
    // 33, 768 43; 4 x 5 tokens on 4,000, of 192 18, 384 24; 8 chunks of up to 100 tokens on 14,000, 512 chunks
    // 112, 768 100.
    // Smaller tiles: 1,024 chunks of 16 rows, 512 of 32, though the chip holds 256 to 1,280 by type and head dim: lengths
    // differ, and a second round of small chunks evens them out.  us with 256, 512, 768, 1,024, 1,280: 4 rows, 64
    // sequences of 4,000 to 16,000, 4 key/value heads, bf16, head dim 128, 256, 245, 248, 227, 229, 64 182, 126, 125, 127,
    // 124, 32 147, 86, 72, 68, 69; fp32, head dim 128, 735, 598, 558, 532, 538.  20 rows, 32 sequences, bf16, head dim 128, 153,
    // 141, 147, 148, 150, 64 95, 64, 66, 70, 69; fp32, head dim 64, 208, 142, 169, 148, 162, 128 442, 389, 376, 395, 388.
    const int64_t wide_held = D == 64 ? 768 : 512;
    int64_t shared_items = 0;
    if (p.stacked) {
        p.all_rows = s.batch * s.rows;
        p.shared_tile = tile_rows_of(p.all_rows, kind.most_shared);
        const int64_t items = (int64_t)s.kv_heads * ((p.all_rows + p.shared_tile - 1) / p.shared_tile);
        const auto splits = [&](int64_t workgroups, int tokens) -> int64_t {
            return workgroups / items < s.prefix_tokens / tokens ? workgroups / items : s.prefix_tokens / tokens;
        };
        int64_t n = splits(wide_held, p.shared_tile == 128 ? 384 : 256);
        // (smaller shares where they leave half of the chip to the own tokens)
        if (p.shared_tile == 128 && n < splits(wide_held / 2, 192)) n = splits(wide_held / 2, 192);
        if (n > 64) n = 64;                            // (what the joining asks for at once)
        p.shared_splits = n < 1 ? 1 : n >= 8 ? (int)n & ~7 : (int)n;
        shared_items = items * p.shared_splits;
    }
    const int64_t tokens = most_tokens(s, p.stacked), units = (tokens + 31) / 32 / (kUnit / 32) + 2;
    const int64_t held = p.tile == 128 || p.shared_tile == 128 ? wide_held : p.tile == 16 ? 1024 : 512;
    if (p.entries <= kMostScanned && p.entries * units < 1 << 30 && (int64_t)p.entries * s.kv_heads < held &&
        tokens >= 384) {
        int64_t n = (held - shared_items) / s.kv_heads;
        if (n < 2 * (int64_t)p.entries) n = 2 * (int64_t)p.entries;
        const int64_t most = p.entries * ((units + kLeast - 1) / kLeast);
        p.chunks = (int)(n < most ? n : most);
    }
    p.scanned = p.chunks > p.entries;
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
