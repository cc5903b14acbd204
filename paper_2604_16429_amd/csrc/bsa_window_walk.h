// The walk of the bf16 matrix-core forward kernels over tiles of 64 keys (head dims 64 and 128).
//
// Four wavefronts with 32 rows each share the tiles, which are gathered straight into LDS.  Per 32
// keys x 32 rows the matrix unit and the exponentials take about the same time, so the two have to
// run side by side inside a wavefront: a step issues the products of the next S^T and of the O^T before
// and spreads the weights of the present tile between them, one weight behind each matrix instruction.
// The fragments of one half of K and one of V are live, read in the step before their use.
//
// One barrier a tile, in the middle of its first step: K of the next tile and V of this one have
// landed then, and the buffers of this K and the V before are free for the gathers of the tiles after,
// which have a whole tile's time.
#pragma once

#include <type_traits>

#include "bsa_window_mfma.h"

namespace bsa {

namespace win {

template <int D>
struct Walk {
    using R = Rows<D>;
    static constexpr int KS = D / 16, DT = D / 32, TILE = R::bytes(64);
    static constexpr int SLOTS = KS + 2 * DT;          // matrix instructions of a step
    static constexpr int PER = 16 / SLOTS;             // weights behind each: 1, at head dim 64 2
    using Tiles = unsigned char[2][2][TILE];           // K, then V: two buffers each
};

// Tiles c_a .. c_e - 1; K of the first two and V of the first have been asked for.  full(c, h): whether all of the
// wavefront's rows see all of half h of tile c (also asked for tile c_e); start(c, h): what its S^T starts
// from otherwise (start_of); issue(c): asks for K of tile c + 2 and V of tile c + 1, as far as there are any.  The
// order of calls: full and start of (c, 1), issue(c), full and start of (c + 1, 0).
template <int D, class Full, class Start, class Issue>
__device__ __forceinline__ void walk_tiles(typename Walk<D>::Tiles& tiles, int c_a, int c_e,
                                           const bf16x8 (&qf)[D / 16], float c2, f32x16 (&acc)[D / 32],
                                           float& m_ref, float& l_run, int lane, Full full, Start start,
                                           Issue issue)
{
    using R = Rows<D>;
    constexpr int KS = Walk<D>::KS, DT = Walk<D>::DT, TILE = Walk<D>::TILE, SLOTS = Walk<D>::SLOTS,
                  PER = Walk<D>::PER;
    // addresses of this lane's fragments: K of the buffer read next, V likewise
    uint32_t k_at[4], v_at[DT], k_other = TILE, v_other = TILE;      // ... and the way to the other one
    R::row_addresses(lds_address(tiles[0][0]), lane, k_at);
    R::trans_addresses(lds_address(tiles[1][0]), lane, v_at);
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
        st[0] = full(c_a, 0) ? splat(0.0f) : start(c_a, 0);
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
        // Weights of half J; S^T of the half after it, of tile `next`; O^T += the half before.
        // `between` runs after the products of S^T and leaves the next fragments of K, `after` those of V.
        auto step = [&](auto J_tag, int next, auto between, auto after) __attribute__((always_inline)) {
            constexpr int J = decltype(J_tag)::value;
            const float neg_m = -m_ref;
            uint32_t w[8];
            float rs0 = 0.0f, rs1 = 0.0f;
            float f[2][2], e[2][2];
            if (full(next, 1 - J))
                st[1 - J] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf[0], qf[0], splat(0.0f), 0, 0, 0);
            else
                st[1 - J] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf[0], qf[0], start(next, 1 - J), 0, 0, 0);
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
            step(std::integral_constant<int, 0>{}, c,
                 [&] {
                     wait_gathers_and_reads();
                     __syncthreads();
                     issue(c);
                     read_k(0);                        // of tile c + 1
                 },
                 [&] { read_v(0); });
            step(std::integral_constant<int, 1>{}, c + 1,
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
}

}  // namespace win

}  // namespace bsa
