// What the kernels of the windowed attention's backward share.
#pragma once

#include "bsa_window.h"

namespace bsa {

namespace win {

constexpr int kKeys = 128;             // keys of a workgroup whose wavefronts share tiles
constexpr float kNoWeight = 3.0e38f;   // lse of a row without keys: its weights are 0

// Sums of the queries beyond the window of the tiles that hold sinks: [slices][groups][chunks + 1][2]
// [32][D] floats, dK (without the scale) and dV of groups of 32 keys; the last ones are those of the
// queries inside the window, where both are made by one launch.
struct Far {
    float* sums;
    int32_t groups, chunks;            // groups of keys that hold sinks (0: no such queries)
    int32_t near_keys;                 // a group's tile is this many keys: 32 or kKeys
};

// Launches of few workgroups share the walk of a workgroup's keys out to `splits` of them, which leave
// sums: [slices][groups of 32 keys][splits][2][32][D] floats, dK (without the scale) and dV.  A kernel
// after them adds these, then the far sums, in their order.
struct Near {
    float* sums;
    int32_t groups, splits;            // splits 1: none
    // tiles first .. end - 1 of `all`, those of split `split`
    __device__ __forceinline__ void share(int split, int all, int& first, int& end) const
    {
        const int per = (all + splits - 1) / splits;
        first = min(all, split * per);
        end = min(all, first + per);
    }
};
template <int D>
__device__ __forceinline__ float* near_part(const Near& near, uint32_t slice, int group, int split, int key)
{
    return near.sums + (((int64_t)slice * near.groups + group) * near.splits + split) * (64 * D) + key * D;
}

// Query tokens a .. e - 1 of a sequence that see keys J .. J + n - 1 inside the window.
struct Span {
    int a, e;
};
__device__ __forceinline__ Span near_span(const Shape& s, int J, int n, int p0, int ql, int kl)
{
    Span t;
    t.a = max(0, J - s.right - p0);
    t.e = J < kl ? min(ql, J + n + s.left - p0) : 0;
    return t;
}
// ... and beyond it (sinks): chunk `chunk` of those.
__device__ __forceinline__ Span far_span(const Shape& s, int J, int n, int p0, int ql, int kl,
                                         int chunk, int chunks)
{
    Span t;
    const int a = max(max(0, J - s.right - p0), J + n + s.left - p0);
    const int all = J < kl ? max(0, ql - a) : 0;
    const int per = ((all + chunks - 1) / chunks + 31) / 32 * 32;
    t.a = a + min(all, chunk * per);
    t.e = a + min(all, (chunk + 1) * per);
    return t;
}
// Whether some query of the sequence sees key j (what no query sees may hold anything).
__device__ __forceinline__ bool is_seen(const Shape& s, int j, int p0, int ql, int kl)
{
    const int last = p0 + ql - 1;
    return j < kl && max(p0, j - s.right) <= (j < s.sinks ? last : min(last, j + s.left));
}

// The queries of a tile that see this lane's key: offsets x of tokens t0 + x with (unsigned)(x -
// first) <= span.
struct Column {
    int first;
    uint32_t span;
    __device__ __forceinline__ bool seen(int x) const { return (uint32_t)(x - first) <= span; }
};
__device__ __forceinline__ Column column(const Shape& s, int j, int kl, int pt0, int tokens)
{
    const int lo = max(0, j - s.right - pt0);
    const int hi = j >= kl ? -1 : min(tokens - 1, j < s.sinks ? tokens : j + s.left - pt0);
    Column c;
    c.first = hi >= lo ? lo : 1 << 20;
    c.span = hi >= lo ? (uint32_t)(hi - lo) : 0u;
    return c;
}

// Adds the far sums of a group of 32 keys to a wavefront's accumulators, in the order of the chunks.
template <int D>
__device__ __forceinline__ void add_far(const Far& far, int64_t slice, int group, int l32, int half,
                                        f32x16 (&ak)[D / 32], f32x16 (&av)[D / 32], float k_sign)
{
    const float* p = far.sums + ((slice * far.groups + group) * (far.chunks + 1)) * (int64_t)(64 * D) + l32 * D;
    for (int c = 0; c < far.chunks; ++c, p += 64 * D) {
#pragma unroll
        for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const f32x4 x = *(const f32x4*)(p + 32 * dt + 8 * r + 4 * half);
                const f32x4 y = *(const f32x4*)(p + 32 * D + 32 * dt + 8 * r + 4 * half);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    ak[dt][4 * r + e] = fmaf(k_sign, x[e], ak[dt][4 * r + e]);
                    av[dt][4 * r + e] += y[e];
                }
            }
    }
}

}  // namespace win

bool window_bwd_mfma_supported(bool is_bf16, int D, const win::Shape& s);
hipError_t launch_window_dq_mfma(int D, const win::Shape& s, const void* q, const void* k,
                                 const void* v, const float* lse, const void* dout, float* delta,
                                 float* lse2, void* dq, hipStream_t stream);
hipError_t launch_window_dkdv_mfma(int D, const win::Shape& s, const void* q, const void* k,
                                   const void* v, const void* dout, const float* delta,
                                   const float* lse2, void* dk, void* dv, const win::Far& far,
                                   const win::Near& near, hipStream_t stream);

}  // namespace bsa
