// Windowed attention backward, bf16, head dims 64 and 128 (see bsa_window_bwd.hip for the formulas
// and the other kernels): dQ, and dK and dV of large launches.
//
// dK and dV: a workgroup of four wavefronts owns 128 keys, 32 to each, and walks the queries that see them
// inside the window, head by head, in tiles of 64 (head dim 128: 32) tokens that are gathered
// straight into LDS, double buffered, one barrier a tile.  Matrix instructions bound it; per 32
// queries x 32 keys there are as many LDS bytes to read as the matrix unit takes time, and
// vector work of about half that time.  So the order of everything in a tile is written out:
// fragments are read several matrix instructions before their use, and the exponentials and
// products of the weights stand behind matrix instructions, two to a slot, where nothing waits
// for the instruction in front of it.  Where the window's border crosses a tile, the products of
// S start from -infinity for what is hidden, so that the order is the same; a wavefront skips
// tiles that none of its keys is seen from.
// At head dim 128 the two accumulators take half of the registers, so V lies in LDS.
#include "bsa_window_bwd.h"
#include "bsa_window_mfma.h"

namespace bsa {

namespace win {

// D = 64: tiles of 64 tokens, V in registers.  D = 128: tiles of 32, V in LDS.  SHARED: the walk is
// shared out.
template <int D, bool SHARED>
__global__ __launch_bounds__(256, 2) void window_dkdv_mfma_kernel(
    const uint16_t* __restrict__ q, const uint16_t* __restrict__ k, const uint16_t* __restrict__ v,
    const uint16_t* __restrict__ dout, const float* __restrict__ delta,
    const float* __restrict__ lse2, uint16_t* __restrict__ dk, uint16_t* __restrict__ dv,
    const Shape s, const Far far, const Near near, uint32_t key_tiles, uint32_t items)
{
    using R = Rows<D>;
    constexpr int KS = D / 16, DT = D / 32, RT = D == 64 ? 64 : 32, TILE = R::bytes(RT);
    constexpr int VB = D == 64 ? 16 : R::bytes(32);     // (no V in LDS at head dim 64)
    using G = Gather<D, RT, 4>;
    // [buffer][Q, dO]
    __shared__ __attribute__((aligned(1024))) unsigned char tiles_s[2][2][TILE];
    __shared__ __attribute__((aligned(1024))) float rows_s[2][2][64];    // [buffer][lse, delta]
    __shared__ __attribute__((aligned(1024))) unsigned char v_s[4][VB];

    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int l32 = lane & 31, half = lane >> 5;

    uint32_t slice;
    int key_tile;
    const int split = SHARED ? (int)(blockIdx.x / items) : 0;
    map_item(s, SHARED ? blockIdx.x - (uint32_t)split * items : blockIdx.x, items, key_tiles, false, slice,
             key_tile);
    const int b = (int)(slice / (uint32_t)s.kv_heads), a = (int)(slice - (uint32_t)b * s.kv_heads);
    int ql, kl;
    lengths(s, b, ql, kl);
    const int p0 = kl - ql;
    const int J = key_tile * kKeys, jw = J + 32 * wave, j = jw + l32;
    const Span span = near_span(s, J, kKeys, p0, ql, kl);
    const int tiles = span.e > span.a ? (span.e - span.a + RT - 1) / RT : 0;
    int it0 = 0, all = tiles * s.group;                 // this workgroup's tiles, head by head
    if (SHARED) near.share(split, all, it0, all);

    auto issue = [&](int head, int t0, int buf) {
        const int n = min(RT, span.e - t0);
        G::gather(q + (int64_t)b * s.q.batch + (int64_t)head * s.q.head + (int64_t)t0 * s.q.token,
                  (uint32_t)s.q.token * 2u, n, lds_address(tiles_s[buf][0]), wave, lane);
        G::gather(dout + (int64_t)b * s.dout.batch + (int64_t)head * s.dout.head +
                      (int64_t)t0 * s.dout.token,
                  (uint32_t)s.dout.token * 2u, n, lds_address(tiles_s[buf][1]), wave, lane);
        const int64_t at = ((int64_t)b * s.heads + head) * s.q_tokens + t0;
        const uint32_t off = (uint32_t)min(lane, n - 1) * 4u;
        if (wave == 0) load_lds_4(buffer_desc(lse2 + at, (uint32_t)n * 4u), off, 0, lds_address(rows_s[buf][0]));
        if (wave == 3) load_lds_4(buffer_desc(delta + at, (uint32_t)n * 4u), off, 0, lds_address(rows_s[buf][1]));
    };
    const int head0 = SHARED && it0 < all ? it0 / tiles : 0;
    int head = a * s.group + head0, t0 = span.a + (it0 - head0 * tiles) * RT;
    if (it0 < all) issue(head, t0, 0);

    // K as operand; -V likewise, or to LDS.  The sign makes delta - dP of a product that starts
    // from delta, so that -dS costs one product; it goes into the scale of dK.
    bf16x8 kf[KS], vf[D == 64 ? KS : 1];
    {
        const bool here = is_seen(s, j, p0, ql, kl);
        const uint16_t* kp = k + (int64_t)b * s.k.batch + (int64_t)a * s.k.head + (int64_t)j * s.k.token + 8 * half;
        const uint16_t* vp = v + (int64_t)b * s.v.batch + (int64_t)a * s.v.head + (int64_t)j * s.v.token + 8 * half;
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
            kf[ks] = here ? *(const bf16x8*)(kp + 16 * ks) : bf16x8{};
            const bf16x8 x = negated(here ? *(const bf16x8*)(vp + 16 * ks) : bf16x8{});
            if constexpr (D == 64) vf[ks] = x;
            else *(bf16x8*)(v_s[wave] + R::place(l32, 2 * ks + half)) = x;
        }
    }
    const float c2 = s.scale * kLog2e;
    f32x16 ak[DT], av[DT];
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) ak[dt] = av[dt] = splat(0.0f);

    // addresses of this lane's fragments in the buffer that is read next
    uint32_t row_at[4], v_at[4], tr_at[DT], val_at = lds_address(rows_s) + 16u * (uint32_t)half;
    R::row_addresses(lds_address(tiles_s), lane, row_at);
    R::row_addresses(lds_address(v_s[wave]), lane, v_at);
    R::trans_addresses(lds_address(tiles_s), lane, tr_at);
    uint32_t to_other = 2u * TILE;                      // from this buffer to the other one
    auto row_frag = [&](int is_g, int row0, int ks) {
        return lds_read<bf16x8>(row_at[R::index(ks)], is_g * TILE + R::bytes(row0) + R::offset(ks));
    };
    auto trans_frag = [&](int is_g, int row0, int dt) {
        return R::trans_frag(tr_at[dt] + (uint32_t)(is_g * TILE), row0);
    };

    // What S starts from in a tile that the window's border crosses: 0, and -infinity where the lane's
    // key does not see the query, which makes the weight 0.
    auto start_of = [&](const Column& col) {
        f32x16 st;
#pragma unroll
        for (int e = 0; e < 16; ++e)
            st[e] = col.seen(8 * (e >> 2) + (e & 3) + 4 * half) ? 0.0f : -INFINITY;
        return st;
    };
    // One tile, D = 64: S, dP of tokens 0..31, then of 32..63 with the weights of the first half
    // behind them, dV, dK of the first half with the weights of the second, dV, dK of the second.
    auto tile64 = [&](bool full, int pa, int n) __attribute__((always_inline)) {
        constexpr int W = 8;                            // fragments read ahead
        auto read_frag = [&](int i) -> bf16x8 {
            const int u = i & 3;
            if (i < 16) return row_frag((i >> 2) & 1, 32 * (i >> 3), u);
            return trans_frag(1 - ((i >> 2) & 1), 32 * ((i - 16) >> 3) + 16 * (u >> 1), u & 1);
        };
        bf16x8 f[W];
        f32x16 st[2], dp[2];
        f32x4 l4[4];
        uint32_t pw[2][8], dw[2][8];
        float fm[2][2], ex[2][2];
        auto read_delta = [&](int qt) {
#pragma unroll
            for (int r4 = 0; r4 < 4; ++r4) {
                const f32x4 d4 = lds_read<f32x4>(val_at, 256 + 128 * qt + 32 * r4);
#pragma unroll
                for (int r = 0; r < 4; ++r) dp[qt][4 * r4 + r] = d4[r];
            }
        };
#pragma unroll
        for (int i = 0; i < 4; ++i) f[i] = read_frag(i);
        read_delta(0);
#pragma unroll
        for (int i = 4; i < W; ++i) f[i] = read_frag(i);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int i = 0; i < 32; ++i) {
            const int u = i & 3;
            const bf16x8 x = f[i % W];
            if (i < 16) {
                const int qt = i >> 3;
                if ((i & 4) == 0 && u > 0)
                    st[qt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(x, kf[u], st[qt], 0, 0, 0);
                else if ((i & 4) == 0 && full)          // (the constant 0 takes no registers)
                    st[qt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(x, kf[u], splat(0.0f), 0, 0, 0);
                else if ((i & 4) == 0)
                    st[qt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(
                        x, kf[u], start_of(column(s, j, kl, pa + 32 * qt, n - 32 * qt)), 0, 0, 0);
                else
                    dp[qt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(x, vf[D == 64 ? u : 0], dp[qt], 0, 0, 0);
            } else {
                const int qt = (i - 16) >> 3, h = u >> 1, dt = u & 1;
                if ((i & 4) == 0)
                    av[dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(x, operand(pw[qt], h), av[dt], 0, 0, 0);
                else
                    ak[dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(x, operand(dw[qt], h), ak[dt], 0, 0, 0);
            }
            if (i + W < 32) f[i % W] = read_frag(i + W);
            // lse of the queries whose weights come next, delta of the second half
            if (i >= 3 && i < 7) l4[i - 3] = lds_read<f32x4>(val_at, 32 * (i - 3));
            if (i == 7) read_delta(1);
            if (i >= 10 && i < 18 && (i & 1) == 0)
                l4[(i - 10) >> 1] = lds_read<f32x4>(val_at, 128 + 32 * ((i - 10) >> 1));
            // two weights to a slot: exponentials, the fma of the next two, products and packs of
            // the two before
            if (i >= 7 && i < 23) {
                const int qt = (i - 7) >> 3, e = 2 * ((i - 7) & 7);
                fm[(i + 1) & 1][0] = fmaf(st[qt][e], c2, -l4[e >> 2][e & 3]);
                fm[(i + 1) & 1][1] = fmaf(st[qt][e + 1], c2, -l4[e >> 2][(e & 3) + 1]);
                asm volatile("" : "+v"(fm[(i + 1) & 1][0]), "+v"(fm[(i + 1) & 1][1]));
            }
            if (i >= 8 && i < 24) {
                ex[i & 1][0] = __builtin_amdgcn_exp2f(fm[i & 1][0]);
                ex[i & 1][1] = __builtin_amdgcn_exp2f(fm[i & 1][1]);
                asm volatile("" : "+v"(ex[i & 1][0]), "+v"(ex[i & 1][1]));
            }
            if (i >= 9 && i < 25) {
                const int qt = (i - 9) >> 3, e = 2 * ((i - 9) & 7), o = (i - 1) & 1;
                pw[qt][e >> 1] = pack_bf16(ex[o][0], ex[o][1]);
                dw[qt][e >> 1] = pack_bf16(ex[o][0] * dp[qt][e], ex[o][1] * dp[qt][e + 1]);
                asm volatile("" : "+v"(pw[qt][e >> 1]), "+v"(dw[qt][e >> 1]));
            }
            __builtin_amdgcn_sched_barrier(0);
        }
    };
    // One tile, D = 128: S, dP, dV, dK; exponentials behind dP, products behind dV.
    auto tile128 = [&](bool full, int pa, int n) __attribute__((always_inline)) {
        constexpr int W = 6;
        // 0-7 Q rows (S), 8-23 dO rows and V in turn (dP), 24-31 dO transposed (dV), 32-39 Q (dK)
        auto read_frag = [&](int i) -> bf16x8 {
            if (i < 8) return row_frag(0, 0, i);
            if (i < 24) {
                const int ks = (i - 8) >> 1;
                if (i & 1) return lds_read<bf16x8>(v_at[R::index(ks)], R::offset(ks));
                return row_frag(1, 0, ks);
            }
            return trans_frag(i < 32, 16 * ((i >> 2) & 1), i & 3);
        };
        bf16x8 f[W];
        f32x16 st, dp;
        f32x4 l4[2];
        uint32_t pw[8], dw[8];
        float fm[2][2];
#pragma unroll
        for (int i = 0; i < W; ++i) f[i] = read_frag(i);
        __builtin_amdgcn_sched_barrier(0);
        auto ask = [&](int i) {
            if (i + W < 40) f[i % W] = read_frag(i + W);
        };
#pragma unroll
        for (int t = 0; t < 32; ++t) {
            const int i = t & 7, h = i >> 2, dt = i & 3;
            if (t == 0) {
                if (full)                               // (the constant 0 takes no registers)
                    st = __builtin_amdgcn_mfma_f32_32x32x16_bf16(f[0], kf[0], splat(0.0f), 0, 0, 0);
                else
                    st = __builtin_amdgcn_mfma_f32_32x32x16_bf16(f[0], kf[0], start_of(column(s, j, kl, pa, n)), 0, 0, 0);
                ask(0);
            } else if (t < 8) {
                st = __builtin_amdgcn_mfma_f32_32x32x16_bf16(f[i % W], kf[i % KS], st, 0, 0, 0);
                ask(i);
            } else if (t < 16) {
                dp = __builtin_amdgcn_mfma_f32_32x32x16_bf16(f[(8 + 2 * i) % W], f[(9 + 2 * i) % W], dp, 0, 0, 0);
                ask(8 + 2 * i);
                ask(9 + 2 * i);
            } else if (t < 24) {
                av[dt % DT] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(f[(24 + i) % W], operand(pw, h), av[dt % DT], 0, 0, 0);
                ask(24 + i);
            } else {
                ak[dt % DT] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(f[(32 + i) % W], operand(dw, h), ak[dt % DT], 0, 0, 0);
                ask(32 + i);
            }
            if (t >= 2 && t < 6) {
                const f32x4 d4 = lds_read<f32x4>(val_at, 256 + 32 * (t - 2));
#pragma unroll
                for (int r = 0; r < 4; ++r) dp[4 * (t - 2) + r] = d4[r];
            }
            if (t == 6 || t == 7) l4[t - 6] = lds_read<f32x4>(val_at, 32 * (t - 6));
            if (t >= 10 && t < 18) {
                const int e = 2 * (t - 10);
                st[e] = __builtin_amdgcn_exp2f(fm[t & 1][0]);
                st[e + 1] = __builtin_amdgcn_exp2f(fm[t & 1][1]);
                pw[e >> 1] = pack_bf16(st[e], st[e + 1]);
                asm volatile("" : "+v"(pw[e >> 1]));
            }
            if (t >= 9 && t < 17) {
                const int e = 2 * (t - 9);
                fm[(t + 1) & 1][0] = fmaf(st[e], c2, -l4[(e >> 2) & 1][e & 3]);
                fm[(t + 1) & 1][1] = fmaf(st[e + 1], c2, -l4[(e >> 2) & 1][(e & 3) + 1]);
                asm volatile("" : "+v"(fm[(t + 1) & 1][0]), "+v"(fm[(t + 1) & 1][1]));
            }
            if (t == 10 || t == 12) l4[(t - 10) >> 1] = lds_read<f32x4>(val_at, 64 + 16 * (t - 10));
            if (t >= 18 && t < 26) {
                const int e = 2 * (t - 18);
                dw[e >> 1] = pack_bf16(st[e] * dp[e], st[e + 1] * dp[e + 1]);
                asm volatile("" : "+v"(dw[e >> 1]));
            }
            __builtin_amdgcn_sched_barrier(0);
        }
    };

    for (int it = it0; it < all; ++it) {
        // tile `it` has landed and everyone is done with the other buffer
        wait_gathers();
        __syncthreads();
        int next_head = head, next_t0 = t0 + RT;
        if (next_t0 >= span.e) { ++next_head; next_t0 = span.a; }
        if (it + 1 < all) issue(next_head, next_t0, (it - it0 + 1) & 1);
        const int n = min(RT, span.e - t0), pa = p0 + t0;
        const bool any = jw < kl && jw <= pa + n - 1 + s.right && (jw + 31 >= pa - s.left || jw < s.sinks);
        const bool full = n == RT && jw + 31 < kl && jw + 31 <= pa + s.right &&
                          (jw >= pa + RT - 1 - s.left || jw + 31 < s.sinks);
        if (any) {
            if constexpr (D == 64) tile64(full, pa, n);
            else tile128(full, pa, n);
        }
        head = next_head;
        t0 = next_t0;
#pragma unroll
        for (int i = 0; i < 4; ++i) row_at[i] += to_other;
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) tr_at[dt] += to_other;
        to_other = 0u - to_other;
        val_at ^= 512u;
    }
    if constexpr (SHARED) {
        if (jw / 32 < near.groups) {
            float* p = near_part<D>(near, slice, jw / 32, split, l32);
            store_lane_row<float, D>(p, ak, -1.0f, half);
            store_lane_row<float, D>(p + 32 * D, av, 1.0f, half);
        }
        return;
    }
    if (jw / 32 < far.groups) add_far<D>(far, slice, jw / 32, l32, half, ak, av, -1.0f);
    if (j < s.k_tokens) {
        store_lane_row<uint16_t, D>(dk + (int64_t)b * s.dk.batch + (int64_t)a * s.dk.head +
                                        (int64_t)j * s.dk.token, ak, -s.scale, half);
        store_lane_row<uint16_t, D>(dv + (int64_t)b * s.dv.batch + (int64_t)a * s.dv.head +
                                        (int64_t)j * s.dv.token, av, 1.0f, half);
    }
}

// delta_i = sum_j P_ij dP_ij of 128 rows, and lse in base 2, for the kernels of dQ, dK and dV: the tiles and
// the two products of the dQ kernel below.  Little but two operands in registers: four wavefronts per SIMD, at head dim
// 128 with tiles of 32 keys.  1.5 degrees, head dim 128, window 1,024: 1,120 us, two wavefronts and tiles of 64 1,180.
template <int D>
__global__ __launch_bounds__(256, 4) void window_delta_mfma_kernel(
    const uint16_t* __restrict__ q, const uint16_t* __restrict__ k, const uint16_t* __restrict__ v,
    const float* __restrict__ lse, const uint16_t* __restrict__ dout, float* __restrict__ delta,
    float* __restrict__ lse2, const Shape s, uint32_t row_tiles, uint32_t items)
{
    using R = Rows<D>;
    constexpr int KS = D / 16, KT = D == 64 ? 64 : 32, TILE = R::bytes(KT);
    using G = KeyGather<D, KT, 4>;
    // [buffer][K, V]
    __shared__ __attribute__((aligned(1024))) unsigned char tiles_s[2][2][TILE];

    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int l32 = lane & 31, half = lane >> 5;

    uint32_t slice;
    int tile_at;
    map_item(s, blockIdx.x, items, row_tiles, true, slice, tile_at);
    const int row0 = tile_at * 128;
    const int b = (int)(slice / (uint32_t)s.kv_heads), a = (int)(slice - (uint32_t)b * s.kv_heads);
    int ql, kl;
    lengths(s, b, ql, kl);
    const int p0 = kl - ql;
    const int t_first = row0 / s.group, t_last = min((row0 + 127) / s.group, ql - 1);
    KeyList keys = {};
    if (t_first <= t_last) keys = key_list(s, p0 + t_first, p0 + t_last, kl);
    const int tiles = (keys.count + KT - 1) / KT;

    const uint32_t k_stride = (uint32_t)s.k.token * 2u, v_stride = (uint32_t)s.v.token * 2u;
    const i32x4 k_rsrc = buffer_desc(k + (int64_t)b * s.k.batch + (int64_t)a * s.k.head,
                                     (uint32_t)(s.k_tokens - 1) * k_stride + R::ROW_BYTES);
    const i32x4 v_rsrc = buffer_desc(v + (int64_t)b * s.v.batch + (int64_t)a * s.v.head,
                                     (uint32_t)(s.k_tokens - 1) * v_stride + R::ROW_BYTES);
    auto issue = [&](int c) {
        G::gather(k_rsrc, k_stride, keys, KT * c, lds_address(tiles_s[c & 1][0]), wave, lane);
        G::gather(v_rsrc, v_stride, keys, KT * c, lds_address(tiles_s[c & 1][1]), wave, lane);
    };
    if (tiles > 0) issue(0);

    const int row = row0 + 32 * wave + l32;
    const int tok = row / s.group, head = a * s.group + (row - tok * s.group);
    const bool valid = row < s.rows && tok < ql;
    const Sight see = sight(s, keys, p0 + tok, kl, valid);
    const RowsSight rows = rows_sight(s, keys, row0 + 32 * wave, 32, p0, ql, kl);
    bf16x8 qf[KS], gf[KS];
    const uint16_t* qp = q + (int64_t)b * s.q.batch + (int64_t)head * s.q.head + (int64_t)tok * s.q.token + 8 * half;
    const uint16_t* gp = dout + (int64_t)b * s.dout.batch + (int64_t)head * s.dout.head +
                         (int64_t)tok * s.dout.token + 8 * half;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
        qf[ks] = valid ? *(const bf16x8*)(qp + 16 * ks) : bf16x8{};
        gf[ks] = valid ? *(const bf16x8*)(gp + 16 * ks) : bf16x8{};
    }
    const int64_t at = ((int64_t)b * s.heads + head) * s.q_tokens + tok;
    const float l = valid ? lse[at] : -INFINITY, l2 = l == -INFINITY ? kNoWeight : l * kLog2e;
    const float c2 = s.scale * kLog2e;
    float d0 = 0.0f, d1 = 0.0f;

    uint32_t row_at[4], to_other = 2u * TILE;
    R::row_addresses(lds_address(tiles_s), lane, row_at);
    for (int c = 0; c < tiles; ++c) {
        // tile c has landed and everyone is done with the other buffer
        wait_gathers();
        __syncthreads();
        if (c + 1 < tiles) issue(c + 1);
#pragma unroll
        for (int hh = 0; hh < KT / 32; ++hh) {
            const int s0 = KT * c + 32 * hh;
            if (!rows.any(s0, 32)) continue;
            f32x16 st = rows.all(s0, 32) ? splat(0.0f) : start_of(see, s0, half, rows.sinks);
            f32x16 dp = splat(0.0f);
#pragma unroll
            for (int ks = 0; ks < KS; ++ks)
                st = __builtin_amdgcn_mfma_f32_32x32x16_bf16(
                    lds_read<bf16x8>(row_at[R::index(ks)], R::bytes(32 * hh) + R::offset(ks)), qf[ks], st, 0, 0, 0);
#pragma unroll
            for (int ks = 0; ks < KS; ++ks)
                dp = __builtin_amdgcn_mfma_f32_32x32x16_bf16(
                    lds_read<bf16x8>(row_at[R::index(ks)], TILE + R::bytes(32 * hh) + R::offset(ks)), gf[ks], dp, 0, 0, 0);
#pragma unroll
            for (int r = 0; r < 16; r += 2) {
                d0 = fmaf(__builtin_amdgcn_exp2f(fmaf(st[r], c2, -l2)), dp[r], d0);
                d1 = fmaf(__builtin_amdgcn_exp2f(fmaf(st[r + 1], c2, -l2)), dp[r + 1], d1);
            }
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) row_at[i] += to_other;
        to_other = 0u - to_other;
    }
    float d = d0 + d1;
    d += swap32(d);
    if (valid && half == 0) {
        delta[at] = d;
        lse2[at] = l2;
    }
}

// dQ of 128 rows: four wavefronts of 32 share tiles of 64 keys, double buffered.
template <int D>
__global__ __launch_bounds__(256, 2) void window_dq_mfma_kernel(
    const uint16_t* __restrict__ q, const uint16_t* __restrict__ k, const uint16_t* __restrict__ v,
    const uint16_t* __restrict__ dout, const float* __restrict__ delta,
    const float* __restrict__ lse2, uint16_t* __restrict__ dq, const Shape s, uint32_t row_tiles, uint32_t items)
{
    using R = Rows<D>;
    constexpr int KS = D / 16, DT = D / 32, TILE = R::bytes(64);
    using G = KeyGather<D, 64, 4>;
    // [buffer][K, V]
    __shared__ __attribute__((aligned(1024))) unsigned char tiles_s[2][2][TILE];

    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int l32 = lane & 31, half = lane >> 5;

    uint32_t slice;
    int tile_at;
    map_item(s, blockIdx.x, items, row_tiles, true, slice, tile_at);
    const int row0 = tile_at * 128;
    const int b = (int)(slice / (uint32_t)s.kv_heads), a = (int)(slice - (uint32_t)b * s.kv_heads);
    int ql, kl;
    lengths(s, b, ql, kl);
    const int p0 = kl - ql;
    const int t_first = row0 / s.group, t_last = min((row0 + 127) / s.group, ql - 1);
    KeyList keys = {};
    if (t_first <= t_last) keys = key_list(s, p0 + t_first, p0 + t_last, kl);
    const int tiles = (keys.count + 63) / 64;

    const uint32_t k_stride = (uint32_t)s.k.token * 2u, v_stride = (uint32_t)s.v.token * 2u;
    const i32x4 k_rsrc = buffer_desc(k + (int64_t)b * s.k.batch + (int64_t)a * s.k.head,
                                     (uint32_t)(s.k_tokens - 1) * k_stride + R::ROW_BYTES);
    const i32x4 v_rsrc = buffer_desc(v + (int64_t)b * s.v.batch + (int64_t)a * s.v.head,
                                     (uint32_t)(s.k_tokens - 1) * v_stride + R::ROW_BYTES);
    auto issue = [&](int c) {
        G::gather(k_rsrc, k_stride, keys, 64 * c, lds_address(tiles_s[c & 1][0]), wave, lane);
        G::gather(v_rsrc, v_stride, keys, 64 * c, lds_address(tiles_s[c & 1][1]), wave, lane);
    };
    if (tiles > 0) issue(0);

    const int row = row0 + 32 * wave + l32;
    const int tok = row / s.group, head = a * s.group + (row - tok * s.group);
    const bool valid = row < s.rows && tok < ql;
    const Sight see = sight(s, keys, p0 + tok, kl, valid);
    const RowsSight rows = rows_sight(s, keys, row0 + 32 * wave, 32, p0, ql, kl);
    bf16x8 qf[KS], gf[KS];
    float neg_l2 = -kNoWeight, neg_delta = 0.0f;
    {
        const uint16_t* qp = q + (int64_t)b * s.q.batch + (int64_t)head * s.q.head + (int64_t)tok * s.q.token + 8 * half;
        const uint16_t* gp = dout + (int64_t)b * s.dout.batch + (int64_t)head * s.dout.head +
                             (int64_t)tok * s.dout.token + 8 * half;
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
            qf[ks] = valid ? *(const bf16x8*)(qp + 16 * ks) : bf16x8{};
            gf[ks] = valid ? *(const bf16x8*)(gp + 16 * ks) : bf16x8{};
        }
        if (valid) {
            const int64_t at = ((int64_t)b * s.heads + head) * s.q_tokens + tok;
            neg_l2 = -lse2[at];
            neg_delta = -delta[at];
        }
    }
    const float c2 = s.scale * kLog2e;
    // dP^T starts from -delta, which leaves one product for dS^T = P^T (dP^T - delta)
    const f32x16 neg_dl = splat(neg_delta);
    f32x16 acc[DT];
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) acc[dt] = splat(0.0f);

    uint32_t row_at[4], tr_at[DT], to_other = 2u * TILE;
    R::row_addresses(lds_address(tiles_s), lane, row_at);
    R::trans_addresses(lds_address(tiles_s), lane, tr_at);
    auto row_frag = [&](int is_v, int r0, int ks) {
        return lds_read<bf16x8>(row_at[R::index(ks)], is_v * TILE + R::bytes(r0) + R::offset(ks));
    };
    auto trans_frag = [&](int r0, int dt) { return R::trans_frag(tr_at[dt], r0); };

    // One tile of 64 keys: S^T and dP^T of both halves, then dQ^T += K^T dS^T of both; behind dP of a
    // half go its exponentials, behind what follows the products.  Fragments are read W ahead.
    auto tile = [&](int slot0) __attribute__((always_inline)) {
        constexpr int W = 8, N = KS, ALL = 4 * N + 4 * DT;       // matrix instructions
        const bool full = rows.all(slot0, 64);
        auto read_frag = [&](int i) -> bf16x8 {
            if (i < 4 * N) return row_frag((i / N) & 1, 32 * (i / (2 * N)), i % N);
            const int u = i - 4 * N;
            return trans_frag(32 * (u / (2 * DT)) + 16 * ((u / DT) & 1), u % DT);
        };
        bf16x8 f[W];
        f32x16 st[2], dp[2];
        uint32_t w[2][8];
        float fm[2][2];
#pragma unroll
        for (int i = 0; i < W; ++i) f[i] = read_frag(i);
        __builtin_amdgcn_sched_barrier(0);
        // two weights to a slot at head dim 128, four at 64: the fma from slot F on, exponentials a
        // slot later, products from slot X on
        constexpr int PER = 16 / N, F = N + 1, X = 2 * N + 2;
        // What S^T of a half starts from.  Head dim 64: its first product stands apart, where the constant 0
        // of a tile without border takes no registers (195 -> 186 us); at 128 the registers that
        // this leaves in the way cost more than 32 moves (1,430 -> 1,700).
        constexpr bool APART = D == 64;
        auto start = [&](int hh) __attribute__((always_inline)) {
            if (!APART) {
                st[hh] = full ? splat(0.0f) : start_of(see, slot0 + 32 * hh, half, rows.sinks);
                return;
            }
            const bf16x8 x = f[(2 * N * hh) % W];
            if (full)
                st[hh] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(x, qf[0], splat(0.0f), 0, 0, 0);
            else
                st[hh] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(
                    x, qf[0], start_of(see, slot0 + 32 * hh, half, rows.sinks), 0, 0, 0);
        };
        auto slot = [&](int t) __attribute__((always_inline)) {
            if (t < 4 * N) {
                const int hh = t / (2 * N), u = t % N;
                if ((t / N) & 1)
                    dp[hh] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(f[t % W], gf[u], u == 0 ? neg_dl : dp[hh], 0, 0, 0);
                else if (!APART || u > 0)
                    st[hh] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(f[t % W], qf[u], st[hh], 0, 0, 0);
            } else {
                const int u = t - 4 * N, hh = u / (2 * DT), h = (u / DT) & 1, dt = u % DT;
                acc[dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(f[t % W], operand(w[hh], h), acc[dt], 0, 0, 0);
            }
            if (t + W < ALL) f[t % W] = read_frag(t + W);
#pragma unroll
            for (int p = 0; p < PER; p += 2) {
                {
                    const int hh = t >= F + 2 * N ? 1 : 0, e = PER * (t - F - 2 * N * hh - 1) + p;
                    if (e >= 0 && e < 16 && t > F) {
                        st[hh][e] = __builtin_amdgcn_exp2f(PER == 2 ? fm[t & 1][0] : st[hh][e]);
                        st[hh][e + 1] = __builtin_amdgcn_exp2f(PER == 2 ? fm[t & 1][1] : st[hh][e + 1]);
                        asm volatile("" : "+v"(st[hh][e]), "+v"(st[hh][e + 1]));
                    }
                }
                {
                    const int hh = t >= F + 2 * N ? 1 : 0, e = PER * (t - F - 2 * N * hh) + p;
                    if (e >= 0 && e < 16) {
                        const float f0 = fmaf(st[hh][e], c2, neg_l2), f1 = fmaf(st[hh][e + 1], c2, neg_l2);
                        if (PER == 2) {
                            fm[(t + 1) & 1][0] = f0;
                            fm[(t + 1) & 1][1] = f1;
                            asm volatile("" : "+v"(fm[(t + 1) & 1][0]), "+v"(fm[(t + 1) & 1][1]));
                        } else {
                            st[hh][e] = f0;
                            st[hh][e + 1] = f1;
                            asm volatile("" : "+v"(st[hh][e]), "+v"(st[hh][e + 1]));
                        }
                    }
                }
                {
                    const int hh = t >= X + 2 * N ? 1 : 0, e = PER * (t - X - 2 * N * hh) + p;
                    if (e >= 0 && e < 16) {
                        w[hh][e >> 1] = pack_bf16(st[hh][e] * dp[hh][e], st[hh][e + 1] * dp[hh][e + 1]);
                        asm volatile("" : "+v"(w[hh][e >> 1]));
                    }
                }
            }
            __builtin_amdgcn_sched_barrier(0);
        };
        start(0);
        if (!APART) start(1);
#pragma unroll
        for (int t = 0; t < 2 * N; ++t) slot(t);
        if (APART) start(1);
#pragma unroll
        for (int t = 2 * N; t < ALL; ++t) slot(t);
    };
    for (int c = 0; c < tiles; ++c) {
        // tile c has landed and everyone is done with the other buffer
        wait_gathers();
        __syncthreads();
        if (c + 1 < tiles) issue(c + 1);
        if (rows.any(64 * c, 64)) tile(64 * c);
#pragma unroll
        for (int i = 0; i < 4; ++i) row_at[i] += to_other;
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) tr_at[dt] += to_other;
        to_other = 0u - to_other;
    }
    __syncthreads();                                    // the tiles are used up
    store_wave_rows<D>(dq + (int64_t)b * s.dq.batch + (int64_t)a * s.group * s.dq.head, s.dq, s,
                       row0 + 32 * wave, acc, s.scale, &tiles_s[0][0][0] + 4096 * wave, lane);
}

}  // namespace win

bool window_bwd_mfma_supported(bool is_bf16, int D, const win::Shape& s)
{
    // 64 rows of a tile are reached by 32-bit offsets
    const int64_t most = (int64_t)1 << 24;
    return is_bf16 && (D == 64 || D == 128) && s.q.token < most && s.dout.token < most &&
           win::slices_fit(s);
}

hipError_t launch_window_dq_mfma(int D, const win::Shape& s, const void* q, const void* k,
                                 const void* v, const float* lse, const void* dout, float* delta,
                                 float* lse2, void* dq, hipStream_t stream)
{
    using namespace win;
    const uint32_t row_tiles = ((uint32_t)s.rows + 127) / 128;
    const uint32_t items = row_tiles * (uint32_t)(s.batch * s.kv_heads);
    auto delta_kernel = D == 64 ? window_delta_mfma_kernel<64> : window_delta_mfma_kernel<128>;
    delta_kernel<<<items, 256, 0, stream>>>((const uint16_t*)q, (const uint16_t*)k, (const uint16_t*)v, lse,
                                            (const uint16_t*)dout, delta, lse2, s, row_tiles, items);
    if (const hipError_t e = hipGetLastError(); e != hipSuccess) return e;
    auto kernel = D == 64 ? window_dq_mfma_kernel<64> : window_dq_mfma_kernel<128>;
    kernel<<<items, 256, 0, stream>>>((const uint16_t*)q, (const uint16_t*)k, (const uint16_t*)v,
                                      (const uint16_t*)dout, delta, lse2, (uint16_t*)dq, s, row_tiles, items);
    return hipGetLastError();
}

hipError_t launch_window_dkdv_mfma(int D, const win::Shape& s, const void* q, const void* k,
                                   const void* v, const void* dout, const float* delta,
                                   const float* lse2, void* dk, void* dv, const win::Far& far,
                                   const win::Near& near, hipStream_t stream)
{
    using namespace win;
    const uint32_t key_tiles = ((uint32_t)s.k_tokens + kKeys - 1) / kKeys;
    const uint32_t items = (uint32_t)(s.batch * s.kv_heads) * key_tiles;
    auto kernel = near.splits > 1 ? (D == 64 ? window_dkdv_mfma_kernel<64, true> : window_dkdv_mfma_kernel<128, true>)
                                  : (D == 64 ? window_dkdv_mfma_kernel<64, false> : window_dkdv_mfma_kernel<128, false>);
    kernel<<<items * (uint32_t)near.splits, 256, 0, stream>>>(
        (const uint16_t*)q, (const uint16_t*)k, (const uint16_t*)v, (const uint16_t*)dout, delta, lse2,
        (uint16_t*)dk, (uint16_t*)dv, s, far, near, key_tiles, items);
    return hipGetLastError();
}

}  // namespace bsa
