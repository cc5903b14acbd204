// Windowed attention forward, bf16, head dims 64 and 128 (see bsa_window_fwd.hip for the others and
// for the joining of parts).
//
// A workgroup of four wavefronts owns 128 rows (token, head of the group), 32 to each, and walks
// the slots of the key list that they share in tiles of 64, gathered straight into LDS.  Per 32
// keys x 32 rows the matrix unit and the exponentials take about the same time, so the two have to
// run side by side inside a wavefront: a step issues the products of the next S^T and of the O^T before
// and spreads the weights of the present tile between them, one weight behind each matrix instruction.
// The fragments of one half of K and one of V are live, read in the step before their use.
//
// One barrier a tile, in the middle of its first step: K of the next tile and V of this one have
// landed then, and the buffers of this K and the V before are free for the gathers of the tiles after,
// which have a whole tile's time.
#include <type_traits>

#include "bsa_window_mfma.h"

namespace bsa {

namespace win {

template <int D>
__global__ __launch_bounds__(256, 2) void window_fwd_mfma_kernel(
    const uint16_t* __restrict__ q, const uint16_t* __restrict__ k, const uint16_t* __restrict__ v,
    uint16_t* __restrict__ out, float* __restrict__ lse, const Shape s, const Parts parts,
    uint32_t row_tiles, uint32_t items)
{
    using R = Rows<D>;
    constexpr int KS = D / 16, DT = D / 32, TILE = R::bytes(64);
    constexpr int SLOTS = KS + 2 * DT;                 // matrix instructions of a step
    constexpr int PER = 16 / SLOTS;                    // weights behind each: 1, at head dim 64 2
    using G = KeyGather<D, 64, 4>;
    // K, then V: two buffers each
    __shared__ __attribute__((aligned(1024))) unsigned char tiles_s[2][2][TILE];

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

    // addresses of this lane's fragments: K of the buffer read next, V likewise
    uint32_t k_at[4], v_at[DT], k_other = TILE, v_other = TILE;      // ... and the way to the other one
    R::row_addresses(lds_address(tiles_s[0][0]), lane, k_at);
    R::trans_addresses(lds_address(tiles_s[1][0]), lane, v_at);
    auto swap_k = [&] {
#pragma unroll
        for (int i = 0; i < 4; ++i) k_at[i] += k_other;
        k_other = 0u - k_other;
    };
    auto swap_v = [&] {
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) v_at[dt] += v_other;
        v_other = 0u - v_other;
    };
    bf16x8 kf[KS], vf[DT][2];
    auto read_k = [&](int hh) {
#pragma unroll
        for (int ks = 0; ks < KS; ++ks)
            kf[ks] = lds_read<bf16x8>(k_at[R::index(ks)], R::bytes(32 * hh) + R::offset(ks));
    };
    auto read_v = [&](int hh) {
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int dt = 0; dt < DT; ++dt) vf[dt][h] = R::trans_frag(v_at[dt], 32 * hh + 16 * h);
    };

    if (c_a < c_e) {
        f32x16 st[2];           // S^T of the halves
        bf16x8 p[2][2];         // their weights
        wait_gathers_and_reads();
        __syncthreads();
        read_k(0);
        st[0] = rows.all(64 * c_a, 32) ? splat(0.0f) : start_of(see, 64 * c_a, half, rows.sinks);
#pragma unroll
        for (int ks = 0; ks < KS; ++ks)
            st[0] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf[ks], qf[ks], st[0], 0, 0, 0);
        __builtin_amdgcn_sched_barrier(0);
        read_k(1);
        swap_k();
        // the first step adds nothing to O
        p[1][0] = p[1][1] = bf16x8{};
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) vf[dt][0] = vf[dt][1] = bf16x8{};

        // a sum of weights out of range: a new reference from the row's maximum
        auto repair = [&](auto J_tag) __attribute__((always_inline)) -> float {
            constexpr int J = decltype(J_tag)::value;
            float mx = st[J][0];
#pragma unroll
            for (int r = 1; r < 16; ++r) mx = fmaxf(mx, st[J][r]);
            mx = fmaxf(mx, swap32(mx));
            const float m_new = fmaxf(m_ref, mx * c2);
            const float alpha = __builtin_amdgcn_exp2f(m_ref - m_new);
            m_ref = m_new;
            l_run *= alpha;
#pragma unroll
            for (int dt = 0; dt < DT; ++dt)
#pragma unroll
                for (int r = 0; r < 16; ++r) acc[dt][r] *= alpha;
            return tile_weights(st[J], c2, -m_new, p[J]);
        };
        // Weights of half J; S^T of the half after it, which starts at `next_slot`; O^T += the half before.
        // `between` runs after the products of S^T and leaves the next fragments of K, `after` those of V.
        auto step = [&](auto J_tag, int next_slot, auto between, auto after) __attribute__((always_inline)) {
            constexpr int J = decltype(J_tag)::value;
            const float neg_m = -m_ref;
            uint32_t w[8];
            float rs0 = 0.0f, rs1 = 0.0f;
            float f[2][2], e[2][2];
            if (rows.all(next_slot, 32))
                st[1 - J] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf[0], qf[0], splat(0.0f), 0, 0, 0);
            else
                st[1 - J] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf[0], qf[0], start_of(see, next_slot, half, rows.sinks), 0, 0, 0);
            f[0][0] = fmaf(st[J][0], c2, neg_m);
            f[0][1] = fmaf(st[J][1], c2, neg_m);
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int t = 0; t < SLOTS; ++t) {
                if (t > 0 && t < KS) {
                    st[1 - J] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf[t], qf[t], st[1 - J], 0, 0, 0);
                } else if (t >= KS) {
                    const int u = t - KS, dt = u % DT, h = u / DT;
                    acc[dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf[dt][h], p[1 - J][h], acc[dt], 0, 0, 0);
                }
                if (t == KS) {
                    between();
                    __builtin_amdgcn_sched_barrier(0);
                }
                // pair x of weights: exponentials, the fma of the next pair, sums and pack of the one before
                if (PER == 2 || t % 2 == 1) {
                    const int x = PER == 2 ? t : t / 2, o = x & 1;
                    e[o][0] = __builtin_amdgcn_exp2f(f[o][0]);
                    e[o][1] = __builtin_amdgcn_exp2f(f[o][1]);
                    if (x + 1 < 8) {
                        f[1 - o][0] = fmaf(st[J][2 * x + 2], c2, neg_m);
                        f[1 - o][1] = fmaf(st[J][2 * x + 3], c2, neg_m);
                        asm volatile("" : "+v"(f[1 - o][0]), "+v"(f[1 - o][1]));
                    }
                    if (x > 0) {
                        w[x - 1] = pack_bf16(e[1 - o][0], e[1 - o][1]);
                        rs0 += e[1 - o][0];
                        rs1 += e[1 - o][1];
                        asm volatile("" : "+v"(w[x - 1]), "+v"(rs0), "+v"(rs1));
                    }
                    asm volatile("" : "+v"(e[o][0]), "+v"(e[o][1]));
                }
                __builtin_amdgcn_sched_barrier(0);
            }
            after();
            w[7] = pack_bf16(e[1][0], e[1][1]);
            rs0 += e[1][0];
            rs1 += e[1][1];
            p[J][0] = __builtin_bit_cast(bf16x8, make_uint4(w[0], w[1], w[2], w[3]));
            p[J][1] = __builtin_bit_cast(bf16x8, make_uint4(w[4], w[5], w[6], w[7]));
            float rs = rs0 + rs1;
            if (__builtin_expect(__builtin_amdgcn_ballot_w64(!(rs <= kSumLimit)) != 0, 0)) rs = repair(J_tag);
            l_run += rs;
        };
        for (int c = c_a; c < c_e; ++c) {
            step(std::integral_constant<int, 0>{}, 64 * c + 32,
                 [&] {
                     wait_gathers_and_reads();
                     __syncthreads();
                     issue_k(c + 2);
                     issue_v(c + 1);
                     read_k(0);                        // of tile c + 1
                 },
                 [&] { read_v(0); });
            step(std::integral_constant<int, 1>{}, 64 * c + 64,
                 [&] {
                     read_k(1);
                     swap_k();
                 },
                 [&] {
                     read_v(1);
                     swap_v();
                 });
        }
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int dt = 0; dt < DT; ++dt)
                acc[dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf[dt][h], p[1][h], acc[dt], 0, 0, 0);
    }

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
