// Windowed attention forward, bf16, head dims 64 and 128 (see bsa_window_fwd.hip for the others and
// for the joining of parts).
//
// A workgroup of four wavefronts owns 128 rows (token, head of the group), 32 to each, and walks
// the slots of the key list that they share in tiles of 64 (bsa_window_walk.h).
#include "bsa_window_walk.h"

namespace bsa {

namespace win {

template <int D>
__global__ __launch_bounds__(256, 2) void window_fwd_mfma_kernel(
    const uint16_t* __restrict__ q, const uint16_t* __restrict__ k, const uint16_t* __restrict__ v,
    uint16_t* __restrict__ out, float* __restrict__ lse, const Shape s, const Parts parts,
    uint32_t row_tiles, uint32_t items)
{
    using R = Rows<D>;
    constexpr int KS = D / 16, DT = D / 32;
    using G = KeyGather<D, 64, 4>;
    __shared__ __attribute__((aligned(1024))) typename Walk<D>::Tiles tiles_s;

    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int l32 = lane & 31, half = lane >> 5;

    const int split = (int)(blockIdx.x % (uint32_t)parts.splits);
    uint32_t slice;
    int tile_at;
    map_item(s, blockIdx.x / (uint32_t)parts.splits, items / (uint32_t)parts.splits, row_tiles, true,
             slice, tile_at);
    const int row0 = tile_at * 128;
    const int b = (int)(slice / (uint32_t)s.kv_heads), a = (int)(slice - (uint32_t)b * s.kv_heads);
    int ql, kl;
    lengths(s, b, ql, kl);
    const int p0 = kl - ql;
    const int t_first = row0 / s.group, t_last = min((row0 + 127) / s.group, ql - 1);
    KeyList keys = {};
    if (t_first <= t_last) keys = key_list(s, p0 + t_first, p0 + t_last, kl);
    int c_a = 0, c_e = (keys.count + 63) / 64;         // this workgroup's tiles
    if (parts.splits > 1) {
        const int per = (c_e + parts.splits - 1) / parts.splits;
        c_a = min(split * per, c_e);
        c_e = min(c_e, c_a + per);
    }

    const uint32_t k_stride = (uint32_t)s.k.token * 2u, v_stride = (uint32_t)s.v.token * 2u;
    const i32x4 k_rsrc = buffer_desc(k + (int64_t)b * s.k.batch + (int64_t)a * s.k.head,
                                     (uint32_t)(s.k_tokens - 1) * k_stride + R::ROW_BYTES);
    const i32x4 v_rsrc = buffer_desc(v + (int64_t)b * s.v.batch + (int64_t)a * s.v.head,
                                     (uint32_t)(s.k_tokens - 1) * v_stride + R::ROW_BYTES);
    auto issue_k = [&](int c) {
        if (c < c_e) G::gather(k_rsrc, k_stride, keys, 64 * c, lds_address(tiles_s[0][(c - c_a) & 1]), wave, lane);
    };
    auto issue_v = [&](int c) {
        if (c < c_e) G::gather(v_rsrc, v_stride, keys, 64 * c, lds_address(tiles_s[1][(c - c_a) & 1]), wave, lane);
    };
    issue_k(c_a);
    issue_v(c_a);
    issue_k(c_a + 1);

    const int row = row0 + 32 * wave + l32;
    const int tok = row / s.group, head = a * s.group + (row - tok * s.group);
    const bool valid = row < s.rows && tok < ql;
    const Sight see = sight(s, keys, p0 + tok, kl, valid);
    const RowsSight rows = rows_sight(s, keys, row0 + 32 * wave, 32, p0, ql, kl);
    bf16x8 qf[KS];
    {
        const uint16_t* p = q + (int64_t)b * s.q.batch + (int64_t)head * s.q.head + (int64_t)tok * s.q.token + 8 * half;
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) qf[ks] = valid ? *(const bf16x8*)(p + 16 * ks) : bf16x8{};
    }
    const float c2 = s.scale * kLog2e;
    f32x16 acc[DT];
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) acc[dt] = splat(0.0f);
    float m_ref = kNoRef, l_run = 0.0f;

    walk_tiles<D>(
        tiles_s, c_a, c_e, qf, c2, acc, m_ref, l_run, lane,
        [&](int c, int h) { return rows.all(64 * c + 32 * h, 32); },
        [&](int c, int h) { return start_of(see, 64 * c + 32 * h, half, rows.sinks); },
        [&](int c) {
            issue_k(c + 2);
            issue_v(c + 1);
        });

    const float l = l_run + swap32(l_run);
    if (parts.splits > 1) {
        if (row < s.rows) {
            const int64_t part = part_of(s, parts, slice, row, split);
            store_lane_row<float, D>(parts.acc + part * D, acc, 1.0f, half);
            if (half == 0) parts.ml[part] = make_float2(m_ref, l);
        }
        return;
    }
    wait_gathers_and_reads();
    __syncthreads();                                   // the tiles are used up
    // (a row that sees nothing: zeros)
    store_wave_rows<D>(out + (int64_t)b * s.out.batch + (int64_t)a * s.group * s.out.head, s.out, s,
                       row0 + 32 * wave, acc, l == 0.0f ? 0.0f : 1.0f / l, &tiles_s[0][0][0] + 4096 * wave,
                       lane);
    if (lse && half == 0 && row < s.rows)
        lse[((int64_t)b * s.heads + head) * s.q_tokens + tok] =
            l == 0.0f ? -INFINITY : (m_ref + __builtin_amdgcn_logf(l)) * kLn2;
}

}  // namespace win

bool window_fwd_mfma_supported(bool is_bf16, int D, const win::Shape& s)
{
    return is_bf16 && (D == 64 || D == 128) && win::slices_fit(s);
}

hipError_t launch_window_fwd_mfma(int D, const win::Shape& s, const void* q, const void* k,
                                  const void* v, void* out, float* lse, const win::Parts& parts,
                                  hipStream_t stream)
{
    using namespace win;
    const uint32_t row_tiles = ((uint32_t)s.rows + 127) / 128;
    const uint32_t items = row_tiles * (uint32_t)(s.batch * s.kv_heads * parts.splits);
    auto kernel = D == 64 ? window_fwd_mfma_kernel<64> : window_fwd_mfma_kernel<128>;
    kernel<<<items, 256, 0, stream>>>((const uint16_t*)q, (const uint16_t*)k, (const uint16_t*)v,
                                      (uint16_t*)out, lse, s, parts, row_tiles, items);
    return hipGetLastError();
}

}  // namespace bsa
