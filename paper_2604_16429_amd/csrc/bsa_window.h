// Windowed attention with sinks: what its kernels share.
//
// Query i of a sequence stands at position p = k_len - q_len + i and sees key j where
//   j < k_len,  j <= p + right  and  (j >= p - left or j < sinks).
// The query heads that share a key/value head are rows of one problem: row r of a
// (batch, key/value head) slice is query token r / group, head r % group.  A tile of rows
// then covers 1 / group as many tokens, so that its keys are fewer and less of them is
// masked, and K and V are fetched once for the whole group.
//
// In bf16 the second product's operands, softmax weights and score gradients, are rounded to bf16,
// which its matrix instruction takes: outputs lie 2.0e-3 to 2.4e-3 (relative 2-norm) from 64 bits, where
// rounding the result alone leaves 1.65e-3.  A second product for what the rounding cuts off would make
// it three products for two.  Scores, sums and statistics are fp32; in fp32 nothing is rounded to less.
#pragma once

#include "bsa_heads.h"
#include "bsa_mfma_common.h"

namespace bsa {

namespace win {

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;
// "no reference yet" of a running softmax, finite so that masked scores (-infinity) weigh 0
// against it
constexpr float kNoRef = -3.0e38f;
constexpr int32_t kUnbounded = 1 << 30;
// Longest sequence that a ring cache may have held, and the bound on a chunk of queries on it: positions
// with a right bound (at most q_tokens) added stay below 2^31.
constexpr int32_t kMostRingLength = 3 << 29, kMostRingChunk = 1 << 28;

struct Shape {
    int32_t batch, heads, kv_heads, group;
    int32_t q_tokens, k_tokens, rows;      // rows = q_tokens * group
    int32_t left, right, sinks, ring;      // left: kUnbounded = no bound; right: at most q_tokens
    float scale;
    const int32_t *q_lens, *k_lens;        // or null
    mosaic_bsa_strides q, k, v, out, dout, dq, dk, dv;    // elements
};

// Lengths of sequence b, held to what the tensors have; b is the same for all lanes, and so
// are the results, in scalar registers with everything that follows from them (a load that a
// kernel's stores might alias would leave them in vector registers).
__device__ __forceinline__ int query_length(const Shape& s, int b)
{
    return s.q_lens ? min(max(s.q_lens[b], 0), s.q_tokens) : s.q_tokens;
}
__device__ __forceinline__ void lengths(const Shape& s, int b, int& ql, int& kl)
{
    ql = __builtin_amdgcn_readfirstlane(query_length(s, b));
    kl = s.k_lens ? min(max(s.k_lens[b], 0), s.ring ? kMostRingLength : s.k_tokens) : s.k_tokens;
    kl = __builtin_amdgcn_readfirstlane(kl);
}

// The keys that queries at positions first .. last see, as slots 0 .. count - 1: `sinks` first
// tokens, then tokens lo, lo + 1, ...
struct KeyList {
    int sinks, lo, count;
    int row_lo, rows, ring;            // row of token lo; rows of the cache
    // Row of k and v that holds a slot's token.  The tokens from lo on are at most `ring`, or none of
    // them is past the first turn of the ring: there is one wrap at most.
    __device__ __forceinline__ int row(int slot) const
    {
        const int r = slot - sinks + row_lo;
        return slot < sinks ? slot : r >= rows ? r - ring : r;
    }
};
__device__ __forceinline__ KeyList key_list(const Shape& s, int first, int last, int kl)
{
    KeyList l;
    const int hi = min(kl - 1, last + s.right);
    l.lo = max(0, first - s.left);
    l.sinks = max(0, min(s.sinks, min(l.lo, hi + 1)));
    l.count = l.sinks + max(0, hi - l.lo + 1);
    l.row_lo = l.lo;
    l.rows = s.k_tokens;
    l.ring = s.ring;
    if (s.ring && l.lo >= s.sinks)
        l.row_lo = s.sinks + (int)((uint32_t)(l.lo - s.sinks) % (uint32_t)s.ring);
    return l;
}

// What one query sees, in slots of a key list that holds all of it: slots below `sinks` and
// those with (unsigned)(slot - first) <= span.
struct Sight {
    int sinks, first;
    uint32_t span;
    __device__ __forceinline__ bool sees(int slot) const
    {
        return slot < sinks || (uint32_t)(slot - first) <= span;
    }
};
__device__ __forceinline__ Sight sight(const Shape& s, const KeyList& keys, int p, int kl, bool valid)
{
    const int hi = valid ? min(kl - 1, p + s.right) : -1, lo = max(0, p - s.left);
    Sight v;
    v.sinks = min(s.sinks, hi + 1);
    v.first = hi >= lo ? lo - keys.lo + keys.sinks : 1 << 30;
    v.span = hi >= lo ? (uint32_t)(hi - lo) : 0u;
    return v;
}

// What rows r0 .. r0 + n - 1 of a slice see: some of them slots below `sinks` and any_a .. any_e, all
// of them all_a .. all_e.
struct RowsSight {
    int sinks, any_a, any_e, all_a, all_e;
    __device__ __forceinline__ bool any(int slot, int n) const
    {
        return slot < sinks || (slot <= any_e && slot + n - 1 >= any_a);
    }
    __device__ __forceinline__ bool all(int slot, int n) const
    {
        return slot >= all_a && slot + n - 1 <= all_e;
    }
};
__device__ __forceinline__ RowsSight rows_sight(const Shape& s, const KeyList& keys, int r0, int n,
                                                int p0, int ql, int kl)
{
    const int first = r0 / s.group, end = (r0 + n - 1) / s.group, last = min(end, ql - 1);
    const int shift = keys.sinks - keys.lo;
    RowsSight v;
    v.any_a = max(0, p0 + first - s.left) + shift;
    v.any_e = first < ql ? min(kl - 1, p0 + last + s.right) + shift : -1;
    v.sinks = first < ql ? min(s.sinks, p0 + last + s.right + 1) : 0;
    v.all_a = max(0, p0 + end - s.left) + shift;
    v.all_e = end < ql && r0 + n <= s.rows ? min(kl - 1, p0 + first + s.right) + shift : -1;
    return v;
}

// Workgroup w of `items` = slices x tiles: which slice and tile it takes.  Workgroups go to the 8 XCDs
// in turn.  Each XCD takes a contiguous eighth of the items, so that tiles with overlapping windows
// meet in one L2.  Where a sequence is shorter than two windows, tiles differ in length: then the
// slices take turns with their longest tiles first (`longest_last`: from the end), which leaves a slice
// to one XCD where 8 divides their number, or to 8 / slices of them.  (16,384 tokens, all before
// visible, 4 slices, forward: eighths 1,290 us.  All XCDs in one slice after the other lose more than
// that balances: 2 x 16 slices of 4,096 tokens, training pass 430 -> 570.)
__device__ __forceinline__ void map_item(const Shape& s, uint32_t w, uint32_t items, uint32_t tiles,
                                         bool longest_last, uint32_t& slice, int& tile)
{
    if (s.left >= s.k_tokens / 2 && s.ring == 0) {
        const uint32_t slices = (uint32_t)(s.batch * s.kv_heads);
        const uint32_t t = w / slices;
        slice = w - t * slices;
        tile = (int)(longest_last ? tiles - 1 - t : t);
        return;
    }
    const uint32_t per = items >> 3, rest = items & 7u, xcd = w & 7u, at = w >> 3;
    const uint32_t item = xcd * per + min(xcd, rest) + at;
    slice = item / tiles;
    tile = (int)(item - slice * tiles);
}

typedef __attribute__((ext_vector_type(8))) float f32x8;

// A 32 x 32 product over 16 channels or keys: a lane holds 8 of them for its row (column),
// lanes 0 .. 31 the first 8, 32 .. 63 the others.  fp32: eight products over two.
template <typename T> struct Mma;
template <> struct Mma<uint16_t> {
    using Frag = bf16x8;
    static __device__ __forceinline__ f32x16 mul(Frag a, Frag b, f32x16 c)
    {
        return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
    }
    static __device__ __forceinline__ Frag load(const uint16_t* p) { return *(const Frag*)p; }
    // weights 8 h .. 8 h + 7 of a tile, rounded (nearest even) to the operand type
    static __device__ __forceinline__ Frag pack(const f32x16& w, int h)
    {
        return __builtin_bit_cast(Frag, make_uint4(pack_bf16(w[8 * h], w[8 * h + 1]),
                                                   pack_bf16(w[8 * h + 2], w[8 * h + 3]),
                                                   pack_bf16(w[8 * h + 4], w[8 * h + 5]),
                                                   pack_bf16(w[8 * h + 6], w[8 * h + 7])));
    }
};
template <> struct Mma<float> {
    using Frag = f32x8;
    static __device__ __forceinline__ f32x16 mul(Frag a, Frag b, f32x16 c)
    {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            c = __builtin_amdgcn_mfma_f32_32x32x2f32(a[i], b[i], c, 0, 0, 0);
        return c;
    }
    static __device__ __forceinline__ Frag load(const float* p)
    {
        const f32x4 x = *(const f32x4*)p, y = *(const f32x4*)(p + 4);
        return __builtin_shufflevector(x, y, 0, 1, 2, 3, 4, 5, 6, 7);
    }
    static __device__ __forceinline__ Frag pack(const f32x16& w, int h)
    {
        Frag f;
#pragma unroll
        for (int i = 0; i < 8; ++i) f[i] = w[8 * h + i];
        return f;
    }
};

// 16 x 16 products over 32 channels or keys: lane l holds 8 of them, from 8 (l / 16) on in the
// order that both operands agree on, for row (column) l % 16.
template <typename T> struct Mma16;
template <> struct Mma16<uint16_t> {
    static __device__ __forceinline__ f32x4 mul(bf16x8 a, bf16x8 b, f32x4 c)
    {
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
    }
    static __device__ __forceinline__ bf16x8 pack(const f32x4& x, const f32x4& y)
    {
        return __builtin_bit_cast(bf16x8, make_uint4(pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3]),
                                                     pack_bf16(y[0], y[1]), pack_bf16(y[2], y[3])));
    }
};
template <> struct Mma16<float> {
    static __device__ __forceinline__ f32x4 mul(f32x8 a, f32x8 b, f32x4 c)
    {
#pragma unroll
        for (int i = 0; i < 8; ++i) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a[i], b[i], c, 0, 0, 0);
        return c;
    }
    static __device__ __forceinline__ f32x8 pack(const f32x4& x, const f32x4& y)
    {
        return __builtin_shufflevector(x, y, 0, 1, 2, 3, 4, 5, 6, 7);
    }
};

// Sum and maximum over the four lanes that hold one row.
__device__ __forceinline__ float row_sum16(float x)
{
    x += __shfl_xor(x, 16);
    return x + swap32(x);
}
__device__ __forceinline__ float row_max16(float x)
{
    x = fmaxf(x, __shfl_xor(x, 16));
    return fmaxf(x, swap32(x));
}

__device__ __forceinline__ f32x16 splat(float x)
{
    f32x16 z;
#pragma unroll
    for (int i = 0; i < 16; ++i) z[i] = x;
    return z;
}

// A tile of ROWS token rows of D channels in LDS, 16-byte chunks swizzled by the row: row
// fragments take the same chunk of 8 consecutive rows, transposing reads a pair of chunks of
// 4 rows.  Filled through registers by THREADS threads, so that the next tile's loads are in
// flight while this one is worked on.
template <typename T, int D, int ROWS, int THREADS = 256>
struct Tile {
    static constexpr int ROW_BYTES = D * sizeof(T);
    static constexpr int CHUNKS = ROW_BYTES / 16;
    static constexpr int BYTES = ROWS * ROW_BYTES;
    static constexpr int PER_THREAD = ROWS * CHUNKS / THREADS;
    static_assert(PER_THREAD >= 1 && ROWS * CHUNKS % THREADS == 0, "whole chunks for every thread");
    using Frag = typename Mma<T>::Frag;

    i32x4 held[PER_THREAD];

    static __device__ __forceinline__ int place(int row, int chunk)
    {
        return row * ROW_BYTES +
               ((chunk ^ ((((row & 3) << 1) | ((row >> 2) & 1)) & (CHUNKS - 1))) << 4);
    }
    // base(row): pointer to that row's first channel, or null: zeros
    template <class F>
    __device__ __forceinline__ void fetch(int tid, F base)
    {
#pragma unroll
        for (int i = 0; i < PER_THREAD; ++i) {
            const int at = tid + THREADS * i, row = at / CHUNKS, chunk = at % CHUNKS;
            const T* p = base(row);
            held[i] = p ? *(const i32x4*)((const char*)p + 16 * chunk) : i32x4{0, 0, 0, 0};
        }
    }
    __device__ __forceinline__ void put(unsigned char* lds, int tid) const
    {
#pragma unroll
        for (int i = 0; i < PER_THREAD; ++i) {
            const int at = tid + THREADS * i;
            *(i32x4*)(lds + place(at / CHUNKS, at % CHUNKS)) = held[i];
        }
    }
    // rows row0 .. row0 + 31 as rows of an operand, channels 16 ks ..
    static __device__ __forceinline__ Frag row_frag(const unsigned char* lds, int row0, int ks,
                                                    int lane)
    {
        const int row = row0 + (lane & 31), half = lane >> 5;
        if constexpr (sizeof(T) == 2) {
            return *(const Frag*)(lds + place(row, 2 * ks + half));
        } else {
            const f32x4 x = *(const f32x4*)(lds + place(row, 4 * ks + 2 * half));
            const f32x4 y = *(const f32x4*)(lds + place(row, 4 * ks + 2 * half + 1));
            return __builtin_shufflevector(x, y, 0, 1, 2, 3, 4, 5, 6, 7);
        }
    }
    // channels 32 dt .. 32 dt + 31 as rows of an operand, the summed index runs over rows row0
    // .. row0 + 15 in the order in which an accumulator's registers hold them
    static __device__ __forceinline__ Frag trans_frag(const unsigned char* lds, int row0, int dt,
                                                      int lane)
    {
        if constexpr (sizeof(T) == 2) {
            const int s16 = lane & 15, gq = lane >> 4;
            const int col = 16 * (gq & 1) + 4 * (s16 & 3) + 32 * dt;
            bf16x4 part[2];
#pragma unroll
            for (int rd = 0; rd < 2; ++rd) {
                const int row = row0 + 8 * rd + 4 * (gq >> 1) + (s16 >> 2);
                const unsigned char* src = lds + place(row, col >> 3) + (col & 7) * 2;
                part[rd] = __builtin_amdgcn_ds_read_tr16_b64_v4bf16(LDS_PTR(bf16x4, src));
            }
            return __builtin_shufflevector(part[0], part[1], 0, 1, 2, 3, 4, 5, 6, 7);
        } else {
            const int d = 32 * dt + (lane & 31), half = lane >> 5;
            Frag f;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int row = row0 + 8 * (i >> 2) + 4 * half + (i & 3);
                f[i] = *(const float*)(lds + place(row, d >> 2) + (d & 3) * 4);
            }
            return f;
        }
    }
};

// Four channels of a row, from accumulator registers.
__device__ __forceinline__ void put4(float* p, float a, float b, float c, float d)
{
    *(float4*)p = make_float4(a, b, c, d);
}
__device__ __forceinline__ void put4(uint16_t* p, float a, float b, float c, float d)
{
    *(uint2*)p = make_uint2(pack_bf16(a, b), pack_bf16(c, d));
}
// A lane's channels 32 dt + 8 r + 4 half + 0..3 of the row at p, times f.
template <typename T, int D>
__device__ __forceinline__ void store_lane_row(T* p, const f32x16 (&acc)[D / 32], float f, int half)
{
#pragma unroll
    for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
        for (int r = 0; r < 4; ++r)
            put4(p + 32 * dt + 8 * r + 4 * half, acc[dt][4 * r] * f, acc[dt][4 * r + 1] * f,
                 acc[dt][4 * r + 2] * f, acc[dt][4 * r + 3] * f);
}

// Few rows: their keys are split over workgroups, each of which leaves what it has of a row
// here, and join_rows adds the parts in their order.
struct Parts {
    float* acc;          // [slices][rows][splits][D]: sum of weight x value against the part's reference
    float2* ml;          // [slices][rows][splits]: reference in base 2, sum of weights
    int32_t splits;      // 1: none
};
__device__ __forceinline__ int64_t part_of(const Shape& s, const Parts& p, uint32_t slice, int row,
                                           int split)
{
    return ((int64_t)slice * s.rows + row) * p.splits + split;
}

// Most keys that `rows` consecutive rows of a slice can see.
inline int64_t most_keys(const Shape& s, int rows)
{
    const int64_t tokens = ((int64_t)rows + s.group - 1) / s.group + 1;
    const int64_t span = (int64_t)s.left + s.right + tokens + s.sinks;
    const int64_t all = s.ring ? (int64_t)s.ring + s.sinks : (int64_t)s.k_tokens;
    return span < all ? span : all;
}
// Up to 16 rows and few keys: as many wavefronts to a workgroup as registers allow, and no parts,
// whose joining is a launch more.
constexpr int step_waves(int element, int D) { return element * D <= 128 ? 16 : element * D <= 256 ? 8 : 4; }
inline bool is_wide_step(bool is_bf16, int D, const Shape& s)
{
    const int waves = step_waves(is_bf16 ? 2 : 4, D);
    return s.rows <= 16 && waves > 4 && most_keys(s, s.rows) <= 128 * waves;
}

}  // namespace win

// Host side: launches, called by the entry points after validation.
hipError_t launch_window_fwd(bool is_bf16, int D, const win::Shape& s, const void* q, const void* k,
                             const void* v, void* out, float* lse, void* workspace,
                             hipStream_t stream);
size_t window_fwd_workspace(bool is_bf16, int D, const win::Shape& s);
hipError_t launch_window_bwd(bool is_bf16, int D, const win::Shape& s, const void* q, const void* k,
                             const void* v, const void* out, const float* lse, const void* dout,
                             void* dq, void* dk, void* dv, void* workspace, hipStream_t stream);
size_t window_bwd_workspace(bool is_bf16, int D, const win::Shape& s);

// bf16 at head dims 64 and 128 in slices that 32-bit offsets reach.
bool window_fwd_mfma_supported(bool is_bf16, int D, const win::Shape& s);
hipError_t launch_window_fwd_mfma(int D, const win::Shape& s, const void* q, const void* k,
                                  const void* v, void* out, float* lse, const win::Parts& parts,
                                  hipStream_t stream);

// Few rows: 16 (all of a slice) or 32 to a workgroup.
hipError_t launch_window_step(bool is_bf16, int D, const win::Shape& s, const void* q, const void* k,
                              const void* v, void* out, float* lse, const win::Parts& parts,
                              hipStream_t stream);

}  // namespace bsa
