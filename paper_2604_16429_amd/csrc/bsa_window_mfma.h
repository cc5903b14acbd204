// Tiles gathered straight into LDS for the windowed attention's bf16 matrix-core kernels.
#pragma once

#include "bsa_window.h"

namespace bsa {

namespace win {

// Rows of D channels in LDS, as one load of a wavefront leaves 1 KiB of them (a slab of 4 or 8 rows).
// LDS serves 16 lanes of 16 bytes at once if they lie in different sixteenths of 256 bytes: lanes 0 to 3, 12 to 15, 20 to
// 23 and 24 to 27 of 32, then the others.  Row fragments take one 16-byte chunk of those rows, transposing
// reads four chunks of 4 rows: a row's chunks are permuted by its place in the slab such that four rows have the
// four in different quarters, and every slab is shifted against the one before, by 16 bytes, at head dim 64, where
// a slab has twice four rows, whose chunks differ by their lowest bit as well, by 32.  (A permutation by the row modulo 8
// alone left half of the LDS cycles in conflicts: 1.5 degrees, head dim 128, window 1,024: forward 1,171 us, dQ
// 1,480, dK/dV 1,990.  Head dim 64 with 16 bytes and the second bit: a third of them, backward 2 to 3 % slower.)
template <int D>
struct Rows {
    static constexpr int ROW_BYTES = 2 * D, CHUNKS = ROW_BYTES / 16, PER_SLAB = 1024 / ROW_BYTES;
    static constexpr int SLAB = 1024 + (D == 64 ? 32 : 16);
    static constexpr int bytes(int rows) { return rows / PER_SLAB * SLAB; }
    static __device__ __forceinline__ int swizzled(int row, int chunk)
    {
        if (D == 128) return chunk ^ ((row & 3) << 2);
        return chunk ^ (((row >> 1) & 1) << 2) ^ ((row >> 2) & 1);
    }
    static __device__ __forceinline__ int place(int row, int chunk)
    {
        return row / PER_SLAB * SLAB + row % PER_SLAB * ROW_BYTES + swizzled(row, chunk) * 16;
    }
    // Fragment ks of a lane's row is at address at[index(ks)] + offset(ks).
    static constexpr int index(int ks) { return D == 128 ? ks >> 1 : ks; }
    static constexpr int offset(int ks) { return D == 128 ? 32 * (ks & 1) : 0; }
    static __device__ __forceinline__ void row_addresses(uint32_t base, int lane, uint32_t (&at)[4])
    {
        const int l32 = lane & 31, half = lane >> 5;
#pragma unroll
        for (int i = 0; i < 4; ++i) at[i] = base + (uint32_t)place(l32, (D == 128 ? 4 : 2) * i + half);
    }
    // Transposing reads: channels 32 dt .., rows 4 (lane / 32) .. + 3 of row0 at at[dt]; 8 rows on for the other
    // half of a fragment.
    static __device__ __forceinline__ void trans_addresses(uint32_t base, int lane, uint32_t (&at)[D / 32])
    {
        const int s16 = lane & 15, gq = lane >> 4, row = 4 * (gq >> 1) + (s16 >> 2);
#pragma unroll
        for (int dt = 0; dt < D / 32; ++dt) {
            const int col = 16 * (gq & 1) + 4 * (s16 & 3) + 32 * dt;
            at[dt] = base + (uint32_t)(place(row, col >> 3) + (col & 7) * 2);
        }
    }
    // rows row0 .. row0 + 15 (a multiple of 16) through at = at[dt]
    static __device__ __forceinline__ bf16x8 trans_frag(uint32_t at, int row0)
    {
        bf16x4 part[2];
#pragma unroll
        for (int rd = 0; rd < 2; ++rd)
            part[rd] = __builtin_amdgcn_ds_read_tr16_b64_v4bf16(
                (__attribute__((address_space(3))) bf16x4*)(uintptr_t)(at + (uint32_t)bytes(row0 + 8 * rd)));
        return __builtin_shufflevector(part[0], part[1], 0, 1, 2, 3, 4, 5, 6, 7);
    }
};

// Tiles of ROWS token rows of one head, gathered into LDS by NW wavefronts: wavefront w takes slabs w +
// NW i, lane l of it chunk l of the slab, for which it fetches the channels that belong there.
template <int D, int ROWS, int NW>
struct Gather {
    using R = Rows<D>;
    static constexpr int LPR = R::CHUNKS, RPS = R::PER_SLAB, MINE = ROWS / RPS / NW;
    // the first n <= ROWS rows from `first` on, of `stride` bytes; rows from n on repeat the last
    static __device__ __forceinline__ void gather(const uint16_t* first, uint32_t stride, int n,
                                                  uint32_t lds, int wave, int lane)
    {
        const i32x4 rsrc = buffer_desc(first, (uint32_t)(n - 1) * stride + R::ROW_BYTES);
        const int x = RPS * wave + lane / LPR;
        const uint32_t chunk = (uint32_t)R::swizzled(lane / LPR, lane % LPR) * 16;
        if (n == ROWS) {
            const uint32_t voff = (uint32_t)x * stride + chunk;
#pragma unroll
            for (int i = 0; i < MINE; ++i)
                load_lds_16(rsrc, voff, (uint32_t)(RPS * NW * i) * stride,
                            lds + (uint32_t)((wave + NW * i) * R::SLAB));
        } else {
#pragma unroll
            for (int i = 0; i < MINE; ++i)
                load_lds_16(rsrc, (uint32_t)min(x + RPS * NW * i, n - 1) * stride + chunk, 0,
                            lds + (uint32_t)((wave + NW * i) * R::SLAB));
        }
    }
};

__device__ __forceinline__ bf16x8 operand(const uint32_t (&w)[8], int h)
{
    return __builtin_bit_cast(bf16x8, make_uint4(w[4 * h], w[4 * h + 1], w[4 * h + 2], w[4 * h + 3]));
}

// Tiles of ROWS slots of a key list, likewise; `rsrc` describes the whole [tokens, D] slice.
template <int D, int ROWS, int NW>
struct KeyGather {
    using R = Rows<D>;
    static constexpr int LPR = R::CHUNKS, RPS = R::PER_SLAB, MINE = ROWS / RPS / NW;
    // slots slot0 .. slot0 + ROWS - 1; those past the list repeat its last
    static __device__ __forceinline__ void gather(i32x4 rsrc, uint32_t stride, const KeyList& keys,
                                                  int slot0, uint32_t lds, int wave, int lane)
    {
        const int x = RPS * wave + lane / LPR;
        const uint32_t chunk = (uint32_t)R::swizzled(lane / LPR, lane % LPR) * 16;
        const int r0 = keys.row(slot0);
        // consecutive rows: nothing but the first row's offset differs from tile to tile
        if (slot0 >= keys.sinks && slot0 + ROWS <= keys.count && r0 + ROWS <= keys.rows) {
            const uint32_t voff = (uint32_t)x * stride + chunk;
#pragma unroll
            for (int i = 0; i < MINE; ++i)
                load_lds_16(rsrc, voff, (uint32_t)(r0 + RPS * NW * i) * stride,
                            lds + (uint32_t)((wave + NW * i) * R::SLAB));
        } else {
#pragma unroll
            for (int i = 0; i < MINE; ++i)
                load_lds_16(rsrc,
                            (uint32_t)keys.row(min(slot0 + x + RPS * NW * i, keys.count - 1)) * stride + chunk,
                            0, lds + (uint32_t)((wave + NW * i) * R::SLAB));
        }
    }
};

// Whether every row of k and v is reached by 32-bit offsets from its slice's start (packed rows of 20 heads of
// 128: up to some 419,000 tokens; the general kernels behind take 1.2 times as long forward at 1.04 M tokens, at
// head dim 128 1.5 times backward).
inline bool slices_fit(const Shape& s)
{
    const int64_t most = ((int64_t)1 << 30) / s.k_tokens;     // elements
    return s.k.token < most && s.v.token < most;
}

// What S^T of a 32 x 32 tile starts from: 0, and -infinity for slots that the lane's query does not
// see, which makes their weights 0.  Slots below `sinks` (of all the wavefront's queries) take one
// comparison more.
__device__ __forceinline__ f32x16 start_of(const Sight& see, int slot0, int half, int sinks)
{
    f32x16 st;
    const uint32_t x = (uint32_t)(slot0 + 4 * half - see.first);
    if (slot0 < sinks) {
        const int y = see.sinks - slot0 - 4 * half;
#pragma unroll
        for (int e = 0; e < 16; ++e) {
            const int c = 8 * (e >> 2) + (e & 3);
            st[e] = x + (uint32_t)c <= see.span || c < y ? 0.0f : -INFINITY;
        }
    } else {
#pragma unroll
        for (int e = 0; e < 16; ++e)
            st[e] = x + (uint32_t)(8 * (e >> 2) + (e & 3)) <= see.span ? 0.0f : -INFINITY;
    }
    return st;
}

// Stores a wavefront's rows row0 .. row0 + 31 (token, head of the group) from accumulators that hold
// a row in the two lanes of its number, times f: through 4 KiB of LDS of its own, 64 channels at a
// time, so that a store instruction writes runs of 128 bytes.  `to`: the batch entry's rows of the first
// head of the group.
template <int D, class S>
__device__ __forceinline__ void store_wave_rows(uint16_t* to, const mosaic_bsa_strides& st, const S& s,
                                                int row0, const f32x16 (&acc)[D / 32], float f,
                                                unsigned char* lds, int lane)
{
    const int l32 = lane & 31, half = lane >> 5;
    uint16_t* row[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int r = row0 + 8 * i + (lane >> 3), tok = r / s.group;
        row[i] = r < s.rows ? to + (int64_t)(r - tok * s.group) * st.head + (int64_t)tok * st.token : nullptr;
    }
#pragma unroll
    for (int c = 0; c < D / 64; ++c) {
#pragma unroll
        for (int dt = 0; dt < 2; ++dt)
#pragma unroll
            for (int r4 = 0; r4 < 4; ++r4) {
                const f32x16& x = acc[2 * c + dt];
                uint2 w;
                w.x = pack_bf16(x[4 * r4] * f, x[4 * r4 + 1] * f);
                w.y = pack_bf16(x[4 * r4 + 2] * f, x[4 * r4 + 3] * f);
                *(uint2*)(lds + l32 * 128 + ((4 * dt + r4) ^ (l32 & 7)) * 16 + 8 * half) = w;
            }
        lane_exchange();
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int t = 8 * i + (lane >> 3);
            const uint4 w = *(const uint4*)(lds + 1024 * i + 16 * lane);
            if (row[i]) *(uint4*)(row[i] + 64 * c + ((lane & 7) ^ (t & 7)) * 8) = w;
        }
        lane_exchange();
    }
}

}  // namespace win

}  // namespace bsa
