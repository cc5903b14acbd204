// Windowed attention forward, any shape the entry point takes, on the matrix cores.
//
// One workgroup of four wavefronts owns 128 rows (token, head of the group) of a (batch,
// key/value head) slice and walks the keys that they see, sinks first, in tiles that all four
// read from LDS.  Per 32 keys x 32 rows: S^T = K Q^T (a lane holds one query and 16 keys), the
// weights against a running reference in fp32, O^T += V^T P^T with the accumulator's registers
// as operand.  The reference moves only when a sum of weights leaves its range.
#include "bsa_window.h"

#include "bsa_launch.h"

namespace bsa {

namespace win {

template <typename T, int D>
__global__ __launch_bounds__(256) void window_fwd_kernel(const T* __restrict__ q,
                                                         const T* __restrict__ k,
                                                         const T* __restrict__ v,
                                                         T* __restrict__ out,
                                                         float* __restrict__ lse, const Shape s,
                                                         const Parts parts, uint32_t row_tiles,
                                                         uint32_t items)
{
    constexpr int KT = sizeof(T) == 2 ? 64 : 32;       // keys of a tile
    constexpr int KS = D / 16, DT = D / 32;
    using Tl = Tile<T, D, KT>;
    using M = Mma<T>;
    using Frag = typename M::Frag;
    __shared__ __attribute__((aligned(1024))) unsigned char k_lds[Tl::BYTES];
    __shared__ __attribute__((aligned(1024))) unsigned char v_lds[Tl::BYTES];

    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
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
    const int p0 = kl - ql;                            // position of query 0

    // this lane's row
    const int row = row0 + 32 * wave + l32;
    const int tok = row / s.group, head = a * s.group + (row - tok * s.group);
    const bool exists = row < s.rows, valid = exists && tok < ql;

    const int t_first = row0 / s.group, t_last = min((row0 + 127) / s.group, ql - 1);
    KeyList keys = {};
    if (t_first <= t_last) keys = key_list(s, p0 + t_first, p0 + t_last, kl);
    const Sight see = sight(s, keys, p0 + tok, kl, valid);
    const RowsSight rows = rows_sight(s, keys, row0 + 32 * wave, 32, p0, ql, kl);

    const T* kb = k + (int64_t)b * s.k.batch + (int64_t)a * s.k.head;
    const T* vb = v + (int64_t)b * s.v.batch + (int64_t)a * s.v.head;

    Frag qf[KS];
    {
        const T* p = q + (int64_t)b * s.q.batch + (int64_t)head * s.q.head + (int64_t)tok * s.q.token;
#pragma unroll
        for (int ks = 0; ks < KS; ++ks)
            qf[ks] = valid ? M::load(p + 16 * ks + 8 * half) : Frag{};
    }
    const float c2 = s.scale * kLog2e;
    f32x16 acc[DT];
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) acc[dt] = splat(0.0f);
    float m_ref = kNoRef, l_run = 0.0f;

    Tl kt, vt;
    auto fetch = [&](int slot0) {
        kt.fetch(tid, [&](int r) -> const T* {
            const int slot = slot0 + r;
            return slot < keys.count ? kb + (int64_t)keys.row(slot) * s.k.token : nullptr;
        });
        vt.fetch(tid, [&](int r) -> const T* {
            const int slot = slot0 + r;
            return slot < keys.count ? vb + (int64_t)keys.row(slot) * s.v.token : nullptr;
        });
    };
    // this workgroup's slots
    int slot_a = 0, slot_e = keys.count;
    if (parts.splits > 1) {
        const int per = ((keys.count + KT - 1) / KT + parts.splits - 1) / parts.splits * KT;
        slot_a = split * per;
        slot_e = min(keys.count, slot_a + per);
    }
    if (slot_a < slot_e) fetch(slot_a);
    for (int slot0 = slot_a; slot0 < slot_e; slot0 += KT) {
        __syncthreads();                               // everyone is done with the tile before
        kt.put(k_lds, tid);
        vt.put(v_lds, tid);
        __syncthreads();
        if (slot0 + KT < slot_e) fetch(slot0 + KT);
#pragma unroll
        for (int hh = 0; hh < KT / 32; ++hh) {
            const int s0 = slot0 + 32 * hh;
            if (s0 >= keys.count || !rows.any(s0, 32)) continue;
            const bool full = rows.all(s0, 32);
            f32x16 st = splat(0.0f);
#pragma unroll
            for (int ks = 0; ks < KS; ++ks)
                st = M::mul(Tl::row_frag(k_lds, 32 * hh, ks, lane), qf[ks], st);
            if (!full) {
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    const int slot = s0 + 8 * (r >> 2) + 4 * half + (r & 3);
                    st[r] = see.sees(slot) ? st[r] : -INFINITY;
                }
            }
            f32x16 w;
            float rs = 0.0f;
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                w[r] = __builtin_amdgcn_exp2f(fmaf(st[r], c2, -m_ref));
                rs += w[r];
            }
            if (__builtin_amdgcn_ballot_w64(!(rs <= kSumLimit)) != 0) {
                float mx = st[0];
#pragma unroll
                for (int r = 1; r < 16; ++r) mx = fmaxf(mx, st[r]);
                mx = fmaxf(mx, swap32(mx));
                const float m_new = fmaxf(m_ref, mx * c2);
                const float alpha = __builtin_amdgcn_exp2f(m_ref - m_new);
                m_ref = m_new;
                l_run *= alpha;
#pragma unroll
                for (int dt = 0; dt < DT; ++dt)
#pragma unroll
                    for (int r = 0; r < 16; ++r) acc[dt][r] *= alpha;
                rs = 0.0f;
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    w[r] = __builtin_amdgcn_exp2f(fmaf(st[r], c2, -m_ref));
                    rs += w[r];
                }
            }
            l_run += rs;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const Frag p = M::pack(w, h);
#pragma unroll
                for (int dt = 0; dt < DT; ++dt)
                    acc[dt] = M::mul(Tl::trans_frag(v_lds, 32 * hh + 16 * h, dt, lane), p, acc[dt]);
            }
        }
    }

    if (!exists) return;
    const float l = l_run + swap32(l_run);
    if (parts.splits > 1) {
        const int64_t part = part_of(s, parts, slice, row, split);
        store_lane_row<float, D>(parts.acc + part * D, acc, 1.0f, half);
        if (half == 0) parts.ml[part] = make_float2(m_ref, l);
        return;
    }
    T* o = out + (int64_t)b * s.out.batch + (int64_t)head * s.out.head + (int64_t)tok * s.out.token;
    // (a row that sees nothing: zeros)
    store_lane_row<T, D>(o, acc, l == 0.0f ? 0.0f : 1.0f / l, half);
    if (lse && half == 0)
        lse[((int64_t)b * s.heads + head) * s.q_tokens + tok] =
            l == 0.0f ? -INFINITY : (m_ref + __builtin_amdgcn_logf(l)) * kLn2;
}

// The parts of a row, in their order: out = sum 2^(m - M) acc / sum 2^(m - M) l.  A thread has
// four channels.
template <typename T, int D>
__global__ __launch_bounds__(256) void window_join_kernel(T* __restrict__ out,
                                                          float* __restrict__ lse, const Shape s,
                                                          const Parts parts, int64_t quads)
{
    const int64_t at = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (at >= quads) return;
    const int c = (int)(at % (D / 4)) * 4;
    const int64_t all_row = at / (D / 4), slice = all_row / s.rows;
    const int row = (int)(all_row - slice * s.rows);
    const float2* ml = parts.ml + all_row * parts.splits;
    const float* acc = parts.acc + all_row * parts.splits * D + c;
    float top = kNoRef;
    for (int i = 0; i < parts.splits; ++i) top = fmaxf(top, ml[i].x);
    float l = 0.0f;
    float4 sum = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    for (int i = 0; i < parts.splits; ++i) {
        const float f = __builtin_amdgcn_exp2f(ml[i].x - top);
        const float4 x = *(const float4*)(acc + (int64_t)i * D);
        l = fmaf(f, ml[i].y, l);
        sum.x = fmaf(f, x.x, sum.x); sum.y = fmaf(f, x.y, sum.y);
        sum.z = fmaf(f, x.z, sum.z); sum.w = fmaf(f, x.w, sum.w);
    }
    const int b = (int)(slice / s.kv_heads), a = (int)(slice - (int64_t)b * s.kv_heads);
    const int tok = row / s.group, head = a * s.group + (row - tok * s.group);
    const float f = l == 0.0f ? 0.0f : 1.0f / l;
    put4(out + (int64_t)b * s.out.batch + (int64_t)head * s.out.head + (int64_t)tok * s.out.token + c,
         sum.x * f, sum.y * f, sum.z * f, sum.w * f);
    if (lse && c == 0)
        lse[((int64_t)b * s.heads + head) * s.q_tokens + tok] =
            l == 0.0f ? -INFINITY : (top + __builtin_amdgcn_logf(l)) * kLn2;
}

// Launches of up to 32 rows, and of fewer workgroups of 128 rows than CUs in fp32 and at head dim 32,
// give 32 rows a workgroup of their own, whose wavefronts share the keys out.  (Nothing here may
// depend on strides, which the size of the workspace is asked for without.)
bool is_step(bool is_bf16, int D, const Shape& s)
{
    return s.rows <= 32 || ((!is_bf16 || D == 32) &&
                            (int64_t)s.batch * s.kv_heads * ((s.rows + 127) / 128) < 256);
}

// Into how many parts the keys of a launch of few workgroups are split: up to 512 workgroups, 256 keys at
// least to each.  Joining costs a launch, so that few keys stay whole, and two or three parts come from 1,280
// keys on.  us, whole | split: bf16, head dim 64, 300 keys 11 | 17, 600 16 | 12, 2,255 45 | 17, 210
// workgroups of 304 10 | 20, of 819 16 | 24, 160 of 1,700, head dim 128, 43 | 35; fp32, head dim 64, 215
// keys 16 | 23, 411 17 | 13.  Parts of 128 keys: 9,830 keys, one token, 18 us instead of 14.  Keys count on both
// sides of a tile: bf16, head dim 64, one head of 3,000 tokens, 63 to the left and all to the right 43 | 19;
// near the borders of the rule up to a third slower (16 slices of 952, head dim 128, 152 and 238 18 | 23).
int splits_of(bool is_bf16, int D, const Shape& s)
{
    const bool step = is_step(is_bf16, D, s);
    if (step && is_wide_step(is_bf16, D, s)) return 1;
    const int tile = !step ? 128 : s.rows <= 16 ? s.rows : 32;
    const int64_t items = (int64_t)s.batch * s.kv_heads * ((s.rows + tile - 1) / tile);
    const int64_t keys = most_keys(s, tile);
    if (keys < (!is_bf16 ? 384 : step ? 640 : 512) || (items > 128 && keys < 1280)) return 1;
    const int64_t n = min(min(512 / items, keys / 256), (int64_t)64);
    return n < 2 ? 1 : (int)n;
}

Parts parts_of(bool is_bf16, int D, const Shape& s, void* workspace)
{
    Parts p = {nullptr, nullptr, splits_of(is_bf16, D, s)};
    if (p.splits > 1) {
        const int64_t n = (int64_t)s.batch * s.kv_heads * s.rows * p.splits;
        p.acc = (float*)workspace;
        p.ml = (float2*)(p.acc + n * D);
    }
    return p;
}

template <typename T, int D>
hipError_t launch(const Shape& s, const void* q, const void* k, const void* v, void* out,
                  float* lse, void* workspace, hipStream_t stream)
{
    const Parts parts = parts_of(sizeof(T) == 2, D, s, workspace);
    hipError_t e;
    if (is_step(sizeof(T) == 2, D, s)) {
        e = launch_window_step(sizeof(T) == 2, D, s, q, k, v, out, lse, parts, stream);
    } else if (window_fwd_mfma_supported(sizeof(T) == 2, D, s)) {
        e = launch_window_fwd_mfma(D, s, q, k, v, out, lse, parts, stream);
    } else {
        const uint32_t row_tiles = ((uint32_t)s.rows + 127) / 128;
        const uint32_t items = row_tiles * (uint32_t)(s.batch * s.kv_heads * parts.splits);
        window_fwd_kernel<T, D><<<items, 256, 0, stream>>>((const T*)q, (const T*)k, (const T*)v,
                                                           (T*)out, lse, s, parts, row_tiles, items);
        e = hipGetLastError();
    }
    if (e != hipSuccess || parts.splits == 1) return e;
    const int64_t quads = (int64_t)s.batch * s.kv_heads * s.rows * (D / 4);
    window_join_kernel<T, D><<<(unsigned)((quads + 255) / 256), 256, 0, stream>>>((T*)out, lse, s,
                                                                                  parts, quads);
    return hipGetLastError();
}

}  // namespace win

size_t window_fwd_workspace(bool is_bf16, int D, const win::Shape& s)
{
    const int splits = win::splits_of(is_bf16, D, s);
    return splits == 1 ? 0 : (size_t)s.batch * s.kv_heads * s.rows * splits * (D + 2) * sizeof(float);
}

hipError_t launch_window_fwd(bool is_bf16, int D, const win::Shape& s, const void* q, const void* k,
                             const void* v, void* out, float* lse, void* workspace,
                             hipStream_t stream)
{
    using namespace win;
#define BSA_WINDOW_FWD(T, D_) win::launch<T, D_>(s, q, k, v, out, lse, workspace, stream)
    if (is_bf16)
        return D == 32   ? BSA_WINDOW_FWD(uint16_t, 32)
               : D == 64 ? BSA_WINDOW_FWD(uint16_t, 64)
                         : BSA_WINDOW_FWD(uint16_t, 128);
    return D == 32   ? BSA_WINDOW_FWD(float, 32)
           : D == 64 ? BSA_WINDOW_FWD(float, 64)
                     : BSA_WINDOW_FWD(float, 128);
#undef BSA_WINDOW_FWD
}

}  // namespace bsa
