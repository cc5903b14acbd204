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
                                                         uint32_t row_tiles, uint32_t items)
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

    const uint32_t item = item_of(blockIdx.x, items);
    const uint32_t slice = item / row_tiles;
    const int row0 = (int)(item - slice * row_tiles) * 128;
    const int b = (int)(slice / (uint32_t)s.kv_heads), a = (int)(slice - (uint32_t)b * s.kv_heads);
    int ql, kl;
    lengths(s, b, ql, kl);
    const int p0 = kl - ql;                            // position of query 0

    // this lane's row
    const int row = row0 + 32 * wave + l32;
    const int tok = row / s.group, head = a * s.group + (row - tok * s.group);
    const bool exists = row < s.rows, valid = exists && tok < ql;
    const Sight see = sight(s, p0 + tok, kl, valid);

    const int t_first = row0 / s.group, t_last = min((row0 + 127) / s.group, ql - 1);
    KeyList keys = {0, 0, 0};
    if (t_first <= t_last) keys = key_list(s, p0 + t_first, p0 + t_last, kl);
    // the same for this wavefront's rows alone
    const int w_first = (row0 + 32 * wave) / s.group, w_end = (row0 + 32 * wave + 31) / s.group;
    const int w_last = min(w_end, ql - 1);
    const int w_lo = p0 + w_first - s.left, w_hi = min(kl - 1, p0 + w_last + s.right);
    const int all_lo = p0 + w_end - s.left, all_hi = min(kl - 1, p0 + w_first + s.right);
    const bool all_valid = w_end < ql && row0 + 32 * wave + 31 < s.rows;

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
            return slot < keys.count ? kb + (int64_t)cache_row(s, keys.token(slot)) * s.k.token : nullptr;
        });
        vt.fetch(tid, [&](int r) -> const T* {
            const int slot = slot0 + r;
            return slot < keys.count ? vb + (int64_t)cache_row(s, keys.token(slot)) * s.v.token : nullptr;
        });
    };
    if (keys.count > 0) fetch(0);
    for (int slot0 = 0; slot0 < keys.count; slot0 += KT) {
        __syncthreads();                               // everyone is done with the tile before
        kt.put(k_lds, tid);
        vt.put(v_lds, tid);
        __syncthreads();
        if (slot0 + KT < keys.count) fetch(slot0 + KT);
#pragma unroll
        for (int hh = 0; hh < KT / 32; ++hh) {
            const int s0 = slot0 + 32 * hh, j0 = s0 - keys.sinks + keys.lo;
            const bool plain = s0 >= keys.sinks;       // all 32 slots are consecutive tokens
            if (s0 >= keys.count || (plain && (j0 > w_hi || (j0 + 31 < w_lo && j0 >= s.sinks))))
                continue;
            const bool full = plain && all_valid && j0 >= all_lo && j0 + 31 <= all_hi;
            f32x16 st = splat(0.0f);
#pragma unroll
            for (int ks = 0; ks < KS; ++ks)
                st = M::mul(Tl::row_frag(k_lds, 32 * hh, ks, lane), qf[ks], st);
            if (!full) {
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    const int slot = s0 + 8 * (r >> 2) + 4 * half + (r & 3);
                    const bool seen = slot < keys.count && see.sees(s, keys.token(slot));
                    st[r] = seen ? st[r] : -INFINITY;
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
    T* o = out + (int64_t)b * s.out.batch + (int64_t)head * s.out.head + (int64_t)tok * s.out.token;
    // (a row that sees nothing: zeros)
    store_lane_row<T, D>(o, acc, l == 0.0f ? 0.0f : 1.0f / l, half);
    if (lse && half == 0)
        lse[((int64_t)b * s.heads + head) * s.q_tokens + tok] =
            l == 0.0f ? -INFINITY : (m_ref + __builtin_amdgcn_logf(l)) * kLn2;
}

template <typename T, int D>
hipError_t launch(const Shape& s, const void* q, const void* k, const void* v, void* out,
                  float* lse, hipStream_t stream)
{
    const uint32_t row_tiles = ((uint32_t)s.rows + 127) / 128;
    const uint32_t items = row_tiles * (uint32_t)(s.batch * s.kv_heads);
    window_fwd_kernel<T, D><<<items, 256, 0, stream>>>((const T*)q, (const T*)k, (const T*)v,
                                                       (T*)out, lse, s, row_tiles, items);
    return hipGetLastError();
}

}  // namespace win

size_t window_fwd_workspace(bool, int, const win::Shape&) { return 0; }

hipError_t launch_window_fwd(bool is_bf16, int D, const win::Shape& s, const void* q, const void* k,
                             const void* v, void* out, float* lse, void* workspace,
                             hipStream_t stream)
{
    using namespace win;
    (void)workspace;
    if (is_bf16)
        return D == 32   ? launch<uint16_t, 32>(s, q, k, v, out, lse, stream)
               : D == 64 ? launch<uint16_t, 64>(s, q, k, v, out, lse, stream)
                         : launch<uint16_t, 128>(s, q, k, v, out, lse, stream);
    return D == 32   ? launch<float, 32>(s, q, k, v, out, lse, stream)
           : D == 64 ? launch<float, 64>(s, q, k, v, out, lse, stream)
                     : launch<float, 128>(s, q, k, v, out, lse, stream);
}

}  // namespace bsa
