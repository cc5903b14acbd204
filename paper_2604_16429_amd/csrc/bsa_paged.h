// Attention over a cache in pages: what its kernels share.
//
// Sequence b has P tokens that all sequences share (the prefix), then kl of its own; its ql queries
// stand at its end.  Query i is token p = P + kl - ql + i and sees token j where
//   j <= p  and  (j >= p - left or j < sinks).
// The query heads that share a key/value head are rows of one problem, as in the windowed attention:
// row r of a (sequence, key/value head) slice is query token r / group, head r % group.
#pragma once

#include "bsa_paged_plan.h"
#include "bsa_window.h"

namespace bsa {

namespace paged {

using win::kLn2;
using win::kLog2e;
using win::kNoRef;
using win::put4;

template <typename T>
struct Args {
    const T *q, *k, *v;
    T* out;
    float* lse;
    Shape s;
    Plan plan;
};

__device__ __forceinline__ int prefix_of(const Shape& s)
{
    return s.prefix_len ? min(max(*s.prefix_len, 0), s.prefix_tokens) : s.prefix_tokens;
}
__device__ __forceinline__ Sequence sequence(const Shape& s, int b)
{
    Sequence q;
    q.ql = s.q_lens ? min(max(s.q_lens[b], 0), s.q_tokens) : s.q_tokens;
    q.kl = min(max(s.k_lens[b], 0), s.table_pages << s.page_shift);
    q.prefix = prefix_of(s);
    return q;
}
// The same for all lanes, in scalar registers.
__device__ __forceinline__ Sequence uniform(const Sequence& q)
{
    return Sequence{__builtin_amdgcn_readfirstlane(q.ql), __builtin_amdgcn_readfirstlane(q.kl),
                    __builtin_amdgcn_readfirstlane(q.prefix)};
}

// The rows that a workgroup owns, from row0 on: of sequence b, or of all sequences one after the other.
struct Rows {
    int row0, n;
    int a, b;                              // key/value head; sequence, or -1: all
};
struct Row {
    int b, tok, head;
    int place;                             // of its query; -1 - tokens: there is no such query
    bool query;
};
// Row `r` of them (r < n); seq: of sequence b.
__device__ __forceinline__ Row row_at(const Shape& s, const Rows& rows, const Sequence& seq, int r)
{
    Row x;
    int row = rows.row0 + r;
    Sequence own = seq;
    x.b = rows.b;
    if (rows.b < 0) {
        x.b = row / s.rows;
        row -= x.b * s.rows;
        own = sequence(s, x.b);
    }
    x.tok = row / s.group;
    x.head = rows.a * s.group + (row - x.tok * s.group);
    x.query = x.tok < own.ql;
    x.place = x.query ? own.prefix + own.kl - own.ql + x.tok : -1;
    return x;
}

// Sum over this lane and those before it, by data-parallel moves: within 16 lanes, then the last of each 16
// (32) lanes into those behind.
__device__ __forceinline__ int wave_scan(int x)
{
#define BSA_SCAN_STEP(CTRL, ROWS) x += __builtin_amdgcn_update_dpp(0, x, CTRL, ROWS, 0xf, false)
    BSA_SCAN_STEP(0x111, 0xf);
    BSA_SCAN_STEP(0x112, 0xf);
    BSA_SCAN_STEP(0x114, 0xf);
    BSA_SCAN_STEP(0x118, 0xf);
    BSA_SCAN_STEP(0x142, 0xa);
    BSA_SCAN_STEP(0x143, 0xc);
#undef BSA_SCAN_STEP
    return x;
}

// Chunk w of a call: its entry, the entry's chunks and the first of them; entry -1: none.  All lanes of a
// wavefront call it with the same w and get the same.  record: entries are written down for the joining.
struct Chunk {
    int entry, first, chunks;
};
__device__ __forceinline__ Chunk chunk_at(const Shape& s, const Plan& plan, int w, int lane, bool record)
{
    constexpr int KEPT = kMostScanned / 64;
    const auto units = [&](int e) -> int {
        return e < plan.entries ? units_of(s, plan, sequence(s, plan.sequence_of(s, e)), plan.tile_of(s, e)) : 0;
    };
    if (!plan.scanned) {
        const int n = plan.stacked ? min(__builtin_amdgcn_readfirstlane(units(w)), 1) : 1;
        if (record && lane == 0) plan.found[w] = Entry{w, n};
        return Chunk{n > 0 ? w : -1, w, 1};
    }
    int kept[KEPT], all = 0;                           // units of the first entries
#pragma unroll
    for (int i = 0; i < KEPT; ++i) {
        kept[i] = 64 * i < plan.entries ? units(64 * i + lane) : 0;
        all += kept[i];
    }
    const auto sum = [&](int x) { return __builtin_amdgcn_readlane(wave_scan(x), 63); };
    const auto chunks = [&](int e, int u, int per) { return e < plan.entries ? chunks_of(plan, u, per) : 0; };
    const int per = chunk_units(plan, sum(all), [&](int c) {
        int n = 0;
#pragma unroll
        for (int i = 0; i < KEPT; ++i) n += chunks(64 * i + lane, kept[i], c);
        return sum(n);
    });
    Chunk found = {-1, 0, 0};
    int run = 0;
#pragma unroll
    for (int i = 0; i < KEPT; ++i) {
        const int base = 64 * i, e = base + lane;
        if (base >= plan.entries) break;
        const int n = chunks(e, kept[i], per);
        const int end = run + wave_scan(n), first = end - n;
        const uint64_t hit = __builtin_amdgcn_ballot_w64(w >= first && w < end);
        if (record && e < plan.entries) plan.found[e] = Entry{first, n};
        if (hit) {
            const int l = __builtin_ctzll(hit);
            found = Chunk{base + l, __builtin_amdgcn_readlane(first, l), __builtin_amdgcn_readlane(n, l)};
            if (!record) break;
        }
        run = __builtin_amdgcn_readlane(end, 63);
    }
    return found;
}

// Four channels of a row's sum against reference `top`: the result, or a part of it.
template <typename T, int D>
__device__ __forceinline__ void store_row(const Args<T>& g, const Row& x, int c, const f32x4& sum, float top, float l)
{
    const Shape& s = g.s;
    const bool none = !x.query || l == 0.0f;
    const float f = 1.0f / l;
    put4(g.out + (int64_t)x.b * s.out.batch + (int64_t)x.head * s.out.head + (int64_t)x.tok * s.out.token + c,
         none ? 0.0f : sum[0] * f, none ? 0.0f : sum[1] * f, none ? 0.0f : sum[2] * f,
         none ? 0.0f : sum[3] * f);
    if (g.lse && c == 0)
        g.lse[((int64_t)x.b * s.heads + x.head) * s.q_tokens + x.tok] =
            none ? -INFINITY : (top + __builtin_amdgcn_logf(l)) * kLn2;
}
template <int D>
__device__ __forceinline__ void store_part(const Plan& plan, int64_t part, int c, const f32x4& sum, float top, float l)
{
    *(f32x4*)(plan.acc + part * D + c) = sum;
    if (c == 0) plan.ml[part] = make_float2(top, l);
}

}  // namespace paged

hipError_t launch_paged_fwd(bool is_bf16, int D, const paged::Shape& s, const void* q, const void* k,
                            const void* v, void* out, float* lse, void* workspace,
                            hipStream_t stream);
size_t paged_fwd_workspace(bool is_bf16, int D, const paged::Shape& s);

}  // namespace bsa
