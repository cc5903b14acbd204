// Tiles gathered straight into LDS for the windowed attention's bf16 matrix-core kernels.
#pragma once

#include "bsa_window.h"

namespace bsa {

namespace win {

__device__ __forceinline__ int swz(int row, int chunk)
{
    return chunk ^ (((row & 3) << 1) | ((row >> 2) & 1));
}

// Tiles of ROWS token rows of one head, gathered into LDS by NW wavefronts: slab wave + NW i is 1 KiB,
// lane l of it fills chunk l and fetches the channels that the swizzle puts there.
template <int D, int ROWS, int NW>
struct Gather {
    static constexpr int ROW_BYTES = 2 * D, LPR = ROW_BYTES / 16, RPS = 1024 / ROW_BYTES;
    static constexpr int BYTES = ROWS * ROW_BYTES, MINE = BYTES / 1024 / NW;
    static_assert(RPS * NW % 8 == 0, "the slabs of a lane share its swizzled chunk");
    // the first n <= ROWS rows from `first` on, of `stride` bytes; rows from n on repeat the last
    static __device__ __forceinline__ void gather(const uint16_t* first, uint32_t stride, int n,
                                                  uint32_t lds, int wave, int lane)
    {
        const i32x4 rsrc = buffer_desc(first, (uint32_t)(n - 1) * stride + ROW_BYTES);
        const int x = RPS * wave + lane / LPR;
        const uint32_t chunk = (uint32_t)swz(x, lane % LPR) * 16;
        if (n == ROWS) {
            const uint32_t voff = (uint32_t)x * stride + chunk;
#pragma unroll
            for (int i = 0; i < MINE; ++i)
                load_lds_16(rsrc, voff, (uint32_t)(RPS * NW * i) * stride,
                            lds + (uint32_t)(wave + NW * i) * 1024u);
        } else {
#pragma unroll
            for (int i = 0; i < MINE; ++i)
                load_lds_16(rsrc, (uint32_t)min(x + RPS * NW * i, n - 1) * stride + chunk, 0,
                            lds + (uint32_t)(wave + NW * i) * 1024u);
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
    static constexpr int ROW_BYTES = 2 * D, LPR = ROW_BYTES / 16, RPS = 1024 / ROW_BYTES;
    static constexpr int BYTES = ROWS * ROW_BYTES, MINE = BYTES / 1024 / NW;
    static_assert(MINE == 1 || RPS * NW % 8 == 0, "the slabs of a lane share its swizzled chunk");
    // slots slot0 .. slot0 + ROWS - 1; those past the list repeat its last
    static __device__ __forceinline__ void gather(i32x4 rsrc, uint32_t stride, const KeyList& keys,
                                                  int slot0, uint32_t lds, int wave, int lane)
    {
        const int x = RPS * wave + lane / LPR;
        const uint32_t chunk = (uint32_t)swz(x, lane % LPR) * 16;
        const int r0 = keys.row(slot0);
        // consecutive rows: nothing but the first row's offset differs from tile to tile
        if (slot0 >= keys.sinks && slot0 + ROWS <= keys.count && r0 + ROWS <= keys.rows) {
            const uint32_t voff = (uint32_t)x * stride + chunk;
#pragma unroll
            for (int i = 0; i < MINE; ++i)
                load_lds_16(rsrc, voff, (uint32_t)(r0 + RPS * NW * i) * stride,
                            lds + (uint32_t)(wave + NW * i) * 1024u);
        } else {
#pragma unroll
            for (int i = 0; i < MINE; ++i)
                load_lds_16(rsrc,
                            (uint32_t)keys.row(min(slot0 + x + RPS * NW * i, keys.count - 1)) * stride + chunk,
                            0, lds + (uint32_t)(wave + NW * i) * 1024u);
        }
    }
};

// Whether every row of k and v is reached by 32-bit offsets from its slice's start.
inline bool slices_fit(const Shape& s)
{
    const int64_t most = ((int64_t)1 << 30) / s.k_tokens;     // elements
    return s.k.token < most && s.v.token < most;
}

// What S^T of a 32 x 32 tile starts from: 0, and -infinity for slots that the lane's query does not
// see, which makes their weights 0.
__device__ __forceinline__ f32x16 start_of(const Sight& see, int slot0, int half)
{
    f32x16 st;
#pragma unroll
    for (int e = 0; e < 16; ++e)
        st[e] = see.sees(slot0 + 8 * (e >> 2) + (e & 3) + 4 * half) ? 0.0f : -INFINITY;
    return st;
}

// Stores a wavefront's rows row0 .. row0 + 31 (token, head of the group) from accumulators that hold
// a row in the two lanes of its number, times f: through 4 KiB of LDS of its own, 64 channels at a
// time, so that a store instruction writes runs of 128 bytes.  `to`: the batch entry's rows of the first
// head of the group.
template <int D>
__device__ __forceinline__ void store_wave_rows(uint16_t* to, const mosaic_bsa_strides& st, const Shape& s,
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
                *(uint2*)(lds + l32 * 128 + swz(l32, 4 * dt + r4) * 16 + 8 * half) = w;
            }
        lane_exchange();
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int t = 8 * i + (lane >> 3);
            const uint4 w = *(const uint4*)(lds + 1024 * i + 16 * lane);
            if (row[i]) *(uint4*)(row[i] + 64 * c + swz(t, lane & 7) * 8) = w;
        }
        lane_exchange();
    }
}

}  // namespace win

}  // namespace bsa
