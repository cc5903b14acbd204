// Windowed attention backward.
//
// With P = exp(scale q.k - lse) recomputed and delta = dO . O for each query,
//   dV_j = sum_i P_ij dO_i    dS_ij = P_ij (dO_i . v_j - delta_i)
//   dQ_i = scale sum_j dS_ij k_j    dK_j = scale sum_i dS_ij q_i
// In bf16 delta is not taken from the rounded output, whose error (and that of the weights it was summed with)
// adds 0.9 to 1.5e-3 to the 2.3e-3 that rounding dS and the results leaves in dQ and dK, more the fewer keys
// share the weight.  With delta' of that output and e = sum_j P_ij (dP_ij - delta'_i), which is delta -
// delta', dQ_i is scale (sum_j dS'_ij k_j - e_i sum_j P_ij k_j); the matrix-core kernels, which have no
// registers for the second sum at head dim 128, take delta = sum_j P_ij dP_ij from a launch before.
//
// Launches: dQ, which walks the keys of 128 rows as the forward does and leaves delta and lse in base
// 2 of each row; dK and dV, where a wavefront owns 32 keys and walks the queries that see them, in tiles
// of consecutive tokens of one head, the heads of the group one after the other.  Every sum has
// one fixed order and no atomics.
//
// A sink is seen by every later query, the keys behind it by window ones: a workgroup that owns
// sinks would walk the whole sequence.  What lies beyond the window of a tile that holds sinks is
// cut into chunks of queries, each with a workgroup of its own that leaves fp32 sums for 32 keys
// in the workspace; the tile's own workgroup, or in small launches a kernel after it, adds them in the
// order of the chunks before it rounds.
#include <algorithm>

#include "bsa_window_bwd.h"

#include "bsa_launch.h"

namespace bsa {

namespace win {

// Wavefronts of a workgroup whose tiles are the wavefronts' own: as many as registers leave room for.
template <typename T, int D>
constexpr int narrow_waves() { return D * (int)sizeof(T) <= 128 ? 8 : 4; }

// The wavefronts' values lane by lane through LDS: those of wavefronts 1 .. are added to wavefront 0's in
// their order.  All wavefronts call it.
template <int NW, int COUNT>
constexpr int add_waves_bytes() { return (NW - 1) * COUNT * 16 * 64 * 4; }
template <int NW, int COUNT>
__device__ __forceinline__ void add_waves(unsigned char* lds, int wave, int lane, f32x16 (&x)[COUNT])
{
    float* const region = (float*)lds + lane;
    __syncthreads();                                    // the tiles (the last values) are used up
    if (wave > 0) {
#pragma unroll
        for (int c = 0; c < COUNT; ++c)
#pragma unroll
            for (int r = 0; r < 16; ++r) region[(((wave - 1) * COUNT + c) * 16 + r) * 64] = x[c][r];
    }
    __syncthreads();
    if (wave > 0) return;
    for (int w = 0; w < NW - 1; ++w)
#pragma unroll
        for (int c = 0; c < COUNT; ++c)
#pragma unroll
            for (int r = 0; r < 16; ++r) x[c][r] += region[((w * COUNT + c) * 16 + r) * 64];
}

// NARROW: the four wavefronts own the same 32 rows and take the tiles of keys in turn, with tiles of
// their own and no barrier between them; else 32 rows each and the tiles are shared.
template <typename T, int D, bool NARROW>
__global__ __launch_bounds__(256, D == 32 ? 3 : 1) void window_dq_kernel(
    const T* __restrict__ q, const T* __restrict__ k, const T* __restrict__ v,
    const T* __restrict__ out, const float* __restrict__ lse, const T* __restrict__ dout,
    float* __restrict__ delta, float* __restrict__ lse2, T* __restrict__ dq, const Shape s,
    uint32_t row_tiles, uint32_t items)
{
    constexpr int KT = sizeof(T) == 2 && !NARROW ? 64 : 32, ROWS = NARROW ? 32 : 128;
    constexpr int KS = D / 16, DT = D / 32, SETS = NARROW ? 4 : 1;
    constexpr bool EXACT = sizeof(T) == 2;              // correct delta by the sum of dS
    using Tl = Tile<T, D, KT, NARROW ? 64 : 256>;
    using M = Mma<T>;
    using Frag = typename M::Frag;
    __shared__ __attribute__((aligned(1024))) unsigned char tiles_s[SETS][2][Tl::BYTES];
    __shared__ float e_s[4][32];
    static_assert(!NARROW || add_waves_bytes<4, DT>() <= (int)sizeof(tiles_s), "the sums fit the tiles");

    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int l32 = lane & 31, half = lane >> 5;
    unsigned char* const k_lds = tiles_s[NARROW ? wave : 0][0];
    unsigned char* const v_lds = tiles_s[NARROW ? wave : 0][1];
    const int loader = NARROW ? lane : tid;

    uint32_t slice;
    int tile_at;
    map_item(s, blockIdx.x, items, row_tiles, true, slice, tile_at);
    const int row0 = tile_at * ROWS;
    const int b = (int)(slice / (uint32_t)s.kv_heads), a = (int)(slice - (uint32_t)b * s.kv_heads);
    int ql, kl;
    lengths(s, b, ql, kl);
    const int p0 = kl - ql;

    const int wave_row = row0 + (NARROW ? 0 : 32 * wave), row = wave_row + l32;
    const int tok = row / s.group, head = a * s.group + (row - tok * s.group);
    const bool exists = row < s.rows, valid = exists && tok < ql;

    const int t_first = row0 / s.group, t_last = min((row0 + ROWS - 1) / s.group, ql - 1);
    KeyList keys = {};
    if (t_first <= t_last) keys = key_list(s, p0 + t_first, p0 + t_last, kl);
    const Sight see = sight(s, keys, p0 + tok, kl, valid);
    const RowsSight rows = rows_sight(s, keys, wave_row, 32, p0, ql, kl);

    const T* kb = k + (int64_t)b * s.k.batch + (int64_t)a * s.k.head;
    const T* vb = v + (int64_t)b * s.v.batch + (int64_t)a * s.v.head;

    Frag qf[KS], gf[KS];
    float neg_l2 = -kNoWeight, neg_delta = 0.0f;
    {
        const T* p = q + (int64_t)b * s.q.batch + (int64_t)head * s.q.head + (int64_t)tok * s.q.token;
        const T* g = dout + (int64_t)b * s.dout.batch + (int64_t)head * s.dout.head +
                     (int64_t)tok * s.dout.token;
        const T* o = out + (int64_t)b * s.out.batch + (int64_t)head * s.out.head +
                     (int64_t)tok * s.out.token;
        float d = 0.0f;
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
            qf[ks] = valid ? M::load(p + 16 * ks + 8 * half) : Frag{};
            gf[ks] = valid ? M::load(g + 16 * ks + 8 * half) : Frag{};
            const Frag of = valid ? M::load(o + 16 * ks + 8 * half) : Frag{};
#pragma unroll
            for (int i = 0; i < 8; ++i) d = fmaf((float)gf[ks][i], (float)of[i], d);
        }
        d += swap32(d);
        if (valid) {
            const int64_t at = ((int64_t)b * s.heads + head) * s.q_tokens + tok;
            const float l = lse[at], l2 = l == -INFINITY ? kNoWeight : l * kLog2e;
            if (half == 0 && (!NARROW || wave == 0)) {
                if (!EXACT) delta[at] = d;
                lse2[at] = l2;
            }
            neg_l2 = -l2;
            neg_delta = -d;
        }
    }
    const float c2 = s.scale * kLog2e;
    f32x16 acc[DT], pk[EXACT ? DT : 1];
    float e_run = 0.0f;
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) acc[dt] = splat(0.0f);
    if constexpr (EXACT) {
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) pk[dt] = splat(0.0f);
    }

    Tl kt, vt;
    auto fetch = [&](int slot0) {
        kt.fetch(loader, [&](int r) -> const T* {
            const int slot = slot0 + r;
            return slot < keys.count ? kb + (int64_t)keys.row(slot) * s.k.token : nullptr;
        });
        vt.fetch(loader, [&](int r) -> const T* {
            const int slot = slot0 + r;
            return slot < keys.count ? vb + (int64_t)keys.row(slot) * s.v.token : nullptr;
        });
    };
    const int first = NARROW ? KT * wave : 0, step = NARROW ? 4 * KT : KT;
    if (first < keys.count) fetch(first);
    for (int slot0 = first; slot0 < keys.count; slot0 += step) {
        if constexpr (NARROW) lane_exchange();
        else __syncthreads();
        kt.put(k_lds, loader);
        vt.put(v_lds, loader);
        if constexpr (NARROW) lane_exchange();
        else __syncthreads();
        if (slot0 + step < keys.count) fetch(slot0 + step);
#pragma unroll
        for (int hh = 0; hh < KT / 32; ++hh) {
            const int s0 = slot0 + 32 * hh;
            if (s0 >= keys.count || !rows.any(s0, 32)) continue;
            const bool full = rows.all(s0, 32);
            f32x16 st = splat(0.0f), dp = splat(neg_delta);
#pragma unroll
            for (int ks = 0; ks < KS; ++ks) {
                st = M::mul(Tl::row_frag(k_lds, 32 * hh, ks, lane), qf[ks], st);
                dp = M::mul(Tl::row_frag(v_lds, 32 * hh, ks, lane), gf[ks], dp);
            }
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                float w = __builtin_amdgcn_exp2f(fmaf(st[r], c2, neg_l2));
                if (!full) {
                    const int slot = s0 + 8 * (r >> 2) + 4 * half + (r & 3);
                    w = see.sees(slot) ? w : 0.0f;
                }
                st[r] = w;
                dp[r] *= w;
                if (EXACT) e_run += dp[r];
            }
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const Frag ds = M::pack(dp, h);
                Frag w;
                if constexpr (EXACT) w = M::pack(st, h);
#pragma unroll
                for (int dt = 0; dt < DT; ++dt) {
                    const Frag x = Tl::trans_frag(k_lds, 32 * hh + 16 * h, dt, lane);
                    acc[dt] = M::mul(x, ds, acc[dt]);
                    if constexpr (EXACT) pk[dt] = M::mul(x, w, pk[dt]);
                }
            }
        }
    }
    float e = e_run + swap32(e_run);
    if constexpr (NARROW) {
        add_waves<4>(&tiles_s[0][0][0], wave, lane, acc);
        if constexpr (EXACT) {
            add_waves<4>(&tiles_s[0][0][0], wave, lane, pk);
            if (half == 0) e_s[wave][l32] = e;
            __syncthreads();
            e = (e_s[0][l32] + e_s[1][l32]) + (e_s[2][l32] + e_s[3][l32]);
        }
        if (wave != 0) return;
    }
    if (!exists) return;
    if constexpr (EXACT) {
#pragma unroll
        for (int dt = 0; dt < DT; ++dt)
#pragma unroll
            for (int r = 0; r < 16; ++r) acc[dt][r] = fmaf(-e, pk[dt][r], acc[dt][r]);
        if (valid && half == 0) delta[((int64_t)b * s.heads + head) * s.q_tokens + tok] = e - neg_delta;
    }
    store_lane_row<T, D>(dq + (int64_t)b * s.dq.batch + (int64_t)head * s.dq.head +
                             (int64_t)tok * s.dq.token,
                         acc, s.scale, half);
}

// The products of 32 keys (operands kf, vf) with 32 queries whose rows lie in LDS; `col`: which of
// them see the lane's key.
template <typename T, int D, class Tl>
__device__ __forceinline__ void key_products(const unsigned char* q_lds, const unsigned char* g_lds,
                                             const float* l2_s, const float* dl_s, int row0, int lane,
                                             const typename Mma<T>::Frag (&kf)[D / 16],
                                             const typename Mma<T>::Frag (&vf)[D / 16], float c2,
                                             bool full, const Column& col, f32x16 (&ak)[D / 32],
                                             f32x16 (&av)[D / 32])
{
    using M = Mma<T>;
    using Frag = typename M::Frag;
    const int half = lane >> 5;
    f32x16 st = splat(0.0f), dp;
#pragma unroll
    for (int r4 = 0; r4 < 4; ++r4) {
        const f32x4 x = *(const f32x4*)(dl_s + 8 * r4 + 4 * half);
#pragma unroll
        for (int e = 0; e < 4; ++e) dp[4 * r4 + e] = -x[e];
    }
#pragma unroll
    for (int ks = 0; ks < D / 16; ++ks) {
        st = M::mul(Tl::row_frag(q_lds, row0, ks, lane), kf[ks], st);
        dp = M::mul(Tl::row_frag(g_lds, row0, ks, lane), vf[ks], dp);
    }
#pragma unroll
    for (int r4 = 0; r4 < 4; ++r4) {
        const f32x4 l = *(const f32x4*)(l2_s + 8 * r4 + 4 * half);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int r = 4 * r4 + e;
            float w = __builtin_amdgcn_exp2f(fmaf(st[r], c2, -l[e]));
            if (!full) w = col.seen(8 * r4 + 4 * half + e) ? w : 0.0f;
            st[r] = w;
            dp[r] *= w;
        }
    }
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const Frag pw = M::pack(st, h), ds = M::pack(dp, h);
#pragma unroll
        for (int dt = 0; dt < D / 32; ++dt) {
            av[dt] = M::mul(Tl::trans_frag(g_lds, row0 + 16 * h, dt, lane), pw, av[dt]);
            ak[dt] = M::mul(Tl::trans_frag(q_lds, row0 + 16 * h, dt, lane), ds, ak[dt]);
        }
    }
}

// K and V of a wavefront's 32 keys as operands; zeros where no query sees a key.
template <typename T, int D>
__device__ __forceinline__ void load_keys(const T* k, const T* v, const Shape& s, int64_t b, int64_t a,
                                          int j, bool here, int half,
                                          typename Mma<T>::Frag (&kf)[D / 16],
                                          typename Mma<T>::Frag (&vf)[D / 16])
{
    using Frag = typename Mma<T>::Frag;
    const T* kp = k + b * s.k.batch + a * s.k.head + (int64_t)j * s.k.token + 8 * half;
    const T* vp = v + b * s.v.batch + a * s.v.head + (int64_t)j * s.v.token + 8 * half;
#pragma unroll
    for (int ks = 0; ks < D / 16; ++ks) {
        kf[ks] = here ? Mma<T>::load(kp + 16 * ks) : Frag{};
        vf[ks] = here ? Mma<T>::load(vp + 16 * ks) : Frag{};
    }
}

// dK and dV of 128 keys, any type and head dim: four wavefronts share the tiles.
template <typename T, int D>
__global__ __launch_bounds__(256) void window_dkdv_kernel(
    const T* __restrict__ q, const T* __restrict__ k, const T* __restrict__ v,
    const T* __restrict__ dout, const float* __restrict__ delta, const float* __restrict__ lse2,
    T* __restrict__ dk, T* __restrict__ dv, const Shape s, const Far far, const Near near,
    uint32_t key_tiles, uint32_t items)
{
    constexpr int RT = sizeof(T) == 2 ? 64 : 32;        // tokens of a tile
    constexpr int KS = D / 16, DT = D / 32;
    using Tl = Tile<T, D, RT>;
    using Frag = typename Mma<T>::Frag;
    __shared__ __attribute__((aligned(1024))) unsigned char q_lds[Tl::BYTES];
    __shared__ __attribute__((aligned(1024))) unsigned char g_lds[Tl::BYTES];
    __shared__ float l2_s[RT], dl_s[RT];

    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int l32 = lane & 31, half = lane >> 5;

    uint32_t slice;
    int key_tile;
    const int split = (int)(blockIdx.x / items);
    map_item(s, blockIdx.x - (uint32_t)split * items, items, key_tiles, false, slice, key_tile);
    const int b = (int)(slice / (uint32_t)s.kv_heads), a = (int)(slice - (uint32_t)b * s.kv_heads);
    int ql, kl;
    lengths(s, b, ql, kl);
    const int p0 = kl - ql;
    const int J = key_tile * kKeys, jw = J + 32 * wave, j = jw + l32;
    const Span span = near_span(s, J, kKeys, p0, ql, kl);

    Frag kf[KS], vf[KS];
    load_keys<T, D>(k, v, s, b, a, j, is_seen(s, j, p0, ql, kl), half, kf, vf);
    const float c2 = s.scale * kLog2e;
    f32x16 ak[DT], av[DT];
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) ak[dt] = av[dt] = splat(0.0f);

    Tl qt, gt;
    float l2_held = 0.0f, dl_held = 0.0f;
    auto fetch = [&](int head, int t0) {
        const T* qb = q + (int64_t)b * s.q.batch + (int64_t)head * s.q.head + (int64_t)t0 * s.q.token;
        const T* gb = dout + (int64_t)b * s.dout.batch + (int64_t)head * s.dout.head +
                      (int64_t)t0 * s.dout.token;
        const int n = span.e - t0;
        qt.fetch(tid, [&](int x) -> const T* { return x < n ? qb + (int64_t)x * s.q.token : nullptr; });
        gt.fetch(tid, [&](int x) -> const T* { return x < n ? gb + (int64_t)x * s.dout.token : nullptr; });
        if (tid < RT) {
            const int64_t at = ((int64_t)b * s.heads + head) * s.q_tokens + t0 + tid;
            l2_held = tid < n ? lse2[at] : kNoWeight;
            dl_held = tid < n ? delta[at] : 0.0f;
        }
    };
    const int tiles = span.e > span.a ? (span.e - span.a + RT - 1) / RT : 0;
    int it0, all;                                       // this workgroup's tiles, head by head
    near.share(split, tiles * s.group, it0, all);
    const int head0 = it0 < all ? it0 / tiles : 0;
    int head = a * s.group + head0, t0 = span.a + (it0 - head0 * tiles) * RT;
    if (it0 < all) fetch(head, t0);
    for (int it = it0; it < all; ++it) {
        __syncthreads();
        qt.put(q_lds, tid);
        gt.put(g_lds, tid);
        if (tid < RT) { l2_s[tid] = l2_held; dl_s[tid] = dl_held; }
        __syncthreads();
        int next_head = head, next_t0 = t0 + RT;
        if (next_t0 >= span.e) { ++next_head; next_t0 = span.a; }
        if (it + 1 < all) fetch(next_head, next_t0);
#pragma unroll
        for (int hh = 0; hh < RT / 32; ++hh) {
            const int ta = t0 + 32 * hh, n = min(32, span.e - ta), pa = p0 + ta;
            if (n <= 0 || jw >= kl || jw > pa + n - 1 + s.right ||
                (jw + 31 < pa - s.left && jw >= s.sinks))
                continue;
            const bool full = n == 32 && jw + 31 < kl && jw + 31 <= pa + s.right &&
                              (jw >= pa + 31 - s.left || jw + 31 < s.sinks);
            key_products<T, D, Tl>(q_lds, g_lds, l2_s + 32 * hh, dl_s + 32 * hh, 32 * hh, lane, kf, vf, c2,
                                   full, column(s, j, kl, pa, n), ak, av);
        }
        head = next_head;
        t0 = next_t0;
    }
    if (near.splits > 1) {
        if (jw / 32 < near.groups) {
            float* p = near_part<D>(near, slice, jw / 32, split, l32);
            store_lane_row<float, D>(p, ak, 1.0f, half);
            store_lane_row<float, D>(p + 32 * D, av, 1.0f, half);
        }
        return;
    }
    if (jw / 32 < far.groups) add_far<D>(far, slice, jw / 32, l32, half, ak, av, 1.0f);
    if (j < s.k_tokens) {
        store_lane_row<T, D>(dk + (int64_t)b * s.dk.batch + (int64_t)a * s.dk.head +
                                 (int64_t)j * s.dk.token, ak, s.scale, half);
        store_lane_row<T, D>(dv + (int64_t)b * s.dv.batch + (int64_t)a * s.dv.head +
                                 (int64_t)j * s.dv.token, av, 1.0f, half);
    }
}

// dK and dV of 32 keys: the wavefronts own the same keys and take the tiles of queries in turn,
// with tiles of their own and no barrier between them; their sums are added in the order of the
// wavefronts.  Workgroups below far_items take one chunk of the queries beyond the window of the tile
// that holds the keys and leave sums in the workspace; the others take those inside the window of
// their group of keys, or a share of them, and leave sums too where it is a share or the keys hold sinks.
template <typename T, int D>
__global__ __launch_bounds__((64 * narrow_waves<T, D>())) void window_dkdv_narrow_kernel(
    const T* __restrict__ q, const T* __restrict__ k, const T* __restrict__ v,
    const T* __restrict__ dout, const float* __restrict__ delta, const float* __restrict__ lse2,
    T* __restrict__ dk, T* __restrict__ dv, const Shape s, const Far far, const Near near,
    uint32_t key_groups, uint32_t far_items, uint32_t near_items)
{
    constexpr int RT = 32, KS = D / 16, DT = D / 32, NW = narrow_waves<T, D>();
    using Tl = Tile<T, D, RT, 64>;
    using Frag = typename Mma<T>::Frag;
    __shared__ __attribute__((aligned(1024))) unsigned char tiles_s[NW][2][Tl::BYTES];
    __shared__ float l2_s[NW][RT], dl_s[NW][RT];
    static_assert(add_waves_bytes<NW, DT>() <= (int)sizeof(tiles_s), "the sums fit the tiles");

    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int l32 = lane & 31, half = lane >> 5;

    const bool is_far = blockIdx.x < far_items;
    const uint32_t chunks = is_far ? (uint32_t)far.chunks : 1u;
    const int split = is_far ? 0 : (int)((blockIdx.x - far_items) / near_items);
    const uint32_t w = is_far ? blockIdx.x / chunks : blockIdx.x - far_items - (uint32_t)split * near_items;
    const int chunk = is_far ? (int)(blockIdx.x - w * chunks) : far.chunks;
    uint32_t slice;
    int group;
    map_item(s, w, is_far ? far_items / chunks : near_items, is_far ? (uint32_t)far.groups : key_groups,
             false, slice, group);
    const int b = (int)(slice / (uint32_t)s.kv_heads), a = (int)(slice - (uint32_t)b * s.kv_heads);
    int ql, kl;
    lengths(s, b, ql, kl);
    const int p0 = kl - ql;
    const int jw = 32 * group, j = jw + l32;
    const Span span = is_far ? far_span(s, jw / far.near_keys * far.near_keys, far.near_keys, p0, ql, kl,
                                        chunk, far.chunks)
                             : near_span(s, jw, 32, p0, ql, kl);

    Frag kf[KS], vf[KS];
    load_keys<T, D>(k, v, s, b, a, j, is_seen(s, j, p0, ql, kl), half, kf, vf);
    const float c2 = s.scale * kLog2e;
    f32x16 ak[DT], av[DT];
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) ak[dt] = av[dt] = splat(0.0f);

    Tl qt, gt;
    float row_held = 0.0f;                              // lse in lanes 0 .. 31, delta in the others
    const int tiles = span.e > span.a ? (span.e - span.a + RT - 1) / RT : 0;
    int it0 = 0, all = tiles * s.group;
    if (!is_far) near.share(split, all, it0, all);
    auto fetch = [&](int it) {
        const int hd = it / tiles, head = a * s.group + hd, t0 = span.a + (it - hd * tiles) * RT;
        const T* qb = q + (int64_t)b * s.q.batch + (int64_t)head * s.q.head + (int64_t)t0 * s.q.token;
        const T* gb = dout + (int64_t)b * s.dout.batch + (int64_t)head * s.dout.head +
                      (int64_t)t0 * s.dout.token;
        const int n = span.e - t0;
        qt.fetch(lane, [&](int x) -> const T* { return x < n ? qb + (int64_t)x * s.q.token : nullptr; });
        gt.fetch(lane, [&](int x) -> const T* { return x < n ? gb + (int64_t)x * s.dout.token : nullptr; });
        const int64_t at = ((int64_t)b * s.heads + head) * s.q_tokens + t0 + l32;
        row_held = l32 < n ? (half ? delta[at] : lse2[at]) : half ? 0.0f : kNoWeight;
    };
    if (it0 + wave < all) fetch(it0 + wave);
    for (int it = it0 + wave; it < all; it += NW) {
        lane_exchange();
        qt.put(tiles_s[wave][0], lane);
        gt.put(tiles_s[wave][1], lane);
        (half ? dl_s : l2_s)[wave][l32] = row_held;
        lane_exchange();
        if (it + NW < all) fetch(it + NW);
        const int t0 = span.a + it % tiles * RT, n = min(RT, span.e - t0), pa = p0 + t0;
        const bool full = n == 32 && jw + 31 < kl && jw + 31 <= pa + s.right &&
                          (jw >= pa + 31 - s.left || jw + 31 < s.sinks);
        key_products<T, D, Tl>(tiles_s[wave][0], tiles_s[wave][1], l2_s[wave], dl_s[wave], 0, lane, kf, vf,
                               c2, full, column(s, j, kl, pa, n), ak, av);
    }
    add_waves<NW>(&tiles_s[0][0][0], wave, lane, ak);
    add_waves<NW>(&tiles_s[0][0][0], wave, lane, av);
    if (wave != 0) return;
    if (!is_far && near.splits > 1) {
        float* p = near_part<D>(near, slice, group, split, l32);
        store_lane_row<float, D>(p, ak, 1.0f, half);
        store_lane_row<float, D>(p + 32 * D, av, 1.0f, half);
    } else if (group < far.groups) {
        float* p = far.sums + (((int64_t)slice * far.groups + group) * (far.chunks + 1) + chunk) * (64 * D) +
                   l32 * D;
        store_lane_row<float, D>(p, ak, 1.0f, half);
        store_lane_row<float, D>(p + 32 * D, av, 1.0f, half);
    } else if (j < s.k_tokens) {
        store_lane_row<T, D>(dk + (int64_t)b * s.dk.batch + (int64_t)a * s.dk.head +
                                 (int64_t)j * s.dk.token, ak, s.scale, half);
        store_lane_row<T, D>(dv + (int64_t)b * s.dv.batch + (int64_t)a * s.dv.head +
                                 (int64_t)j * s.dv.token, av, 1.0f, half);
    }
}

// dK and dV of the first `groups` groups of 32 keys of each slice: shares of the near walk in their
// order, if there are any, then the far sums of groups that hold sinks in the order of the chunks (the
// last of which is the near walk where that is not shared out).  A thread has four channels.
template <typename T, int D>
__global__ __launch_bounds__(256) void window_keys_kernel(T* __restrict__ dk, T* __restrict__ dv,
                                                          const Shape s, const Far far, const Near near,
                                                          int groups, int64_t quads)
{
    const int64_t at = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (at >= quads) return;
    const int in_part = (int)(at % (16 * D)) * 4;       // [2][32][D]
    const int64_t which = at / (16 * D), slice = which / groups;
    const int is_v = in_part / (32 * D), key = in_part / D % 32, c = in_part % D;
    const int group = (int)(which - slice * groups), j = group * 32 + key;
    if (j >= s.k_tokens) return;
    float4 sum = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    auto add = [&](const float* p, int n) __attribute__((always_inline)) {
#pragma unroll 8
        for (int i = 0; i < n; ++i) {
            const float4 x = *(const float4*)(p + (int64_t)i * (64 * D));
            sum.x += x.x; sum.y += x.y; sum.z += x.z; sum.w += x.w;
        }
    };
    const bool shared = near.splits > 1;
    if (shared) add(near_part<D>(near, (uint32_t)slice, group, 0, 0) + in_part, near.splits);
    if (group < far.groups)
        add(far.sums + (slice * far.groups + group) * (far.chunks + 1) * (64 * D) + in_part,
            far.chunks + (shared ? 0 : 1));
    const int b = (int)(slice / s.kv_heads), a = (int)(slice - (int64_t)b * s.kv_heads);
    if (is_v)
        store4(dv + (int64_t)b * s.dv.batch + (int64_t)a * s.dv.head + (int64_t)j * s.dv.token + c, sum);
    else
        store4(dk + (int64_t)b * s.dk.batch + (int64_t)a * s.dk.head + (int64_t)j * s.dk.token + c,
               make_float4(sum.x * s.scale, sum.y * s.scale, sum.z * s.scale, sum.w * s.scale));
}

size_t rounded(size_t x) { return (x + 255) & ~(size_t)255; }

size_t row_bytes(const Shape& s)
{
    return rounded((size_t)s.batch * s.kv_heads * s.rows * sizeof(float));
}

// How dK and dV are launched.
struct Plan {
    bool narrow;                       // 32 keys a workgroup
    Far far;
    Near near;
    size_t far_bytes, near_bytes;
};

// Few workgroups of 128 keys: every 32 keys get one of their own.  Four query heads to a key head, us,
// narrow | not: 120 workgroups, head dim 64, windows 64 and 300 32 | 43 and 40 | 65; from 128 on, whole
// training pass, head dim 128, window 700: 142 334 | 289, 204 425 | 326.
//
// Where that leaves CUs idle, or one round and a bit of workgroups, the walk is shared out.  us, whole |
// shared: under 256 workgroups, up to 512 shares of 4 tiles at least: head dim 128, window 641, 237 191 |
// 114, both sides 1,555, 196 579 | 456, head dim 64, window 219, 184 95 | 77; 256 to 511 (any number in
// the kernels without an order of their own), up to 2,048 of 16 tiles (24 with one): head dim 64, both sides 2,577, 354
// 1,157 | 1,033, fp32, head dim 32, window 482, 944 2,800 | 2,460 (with shares of 4 tiles: head dim 128,
// window 56, 295 92 | 124; with an order of their own, 840 workgroups 557 | 633).
Plan plan_of(bool mfma, int element, int D, const Shape& s)
{
    Plan p;
    const int64_t slices = (int64_t)s.batch * s.kv_heads, groups = ((int64_t)s.k_tokens + 31) / 32;
    const int64_t key_tiles = slices * (((int64_t)s.k_tokens + kKeys - 1) / kKeys);
    p.narrow = key_tiles < (mfma ? 128 : 256);
    // shares of workgroups with n keys: at least `least` tiles of `rows` queries to each
    auto shares = [&](int64_t room, int64_t workgroups, int n, int rows, int least) {
        const int64_t left = min(s.left, s.k_tokens), right = min(s.right, s.k_tokens);
        const int64_t walk = min((int64_t)s.q_tokens, left + right + n);
        const int64_t tiles = (walk + rows - 1) / rows * s.group;
        return (int)max((int64_t)1, min(min(room / workgroups, tiles / least), (int64_t)32));
    };
    int splits;
    if (p.narrow) {
        const int waves = D * element <= 128 ? 8 : 4;
        splits = shares(256, slices * groups, 32, 32, 2 * waves);
    } else {
        const int rows = element == 4 || (mfma && D == 128) ? 32 : 64;
        splits = key_tiles < 256            ? shares(512, key_tiles, kKeys, rows, 4)
                 : mfma && key_tiles >= 512 ? 1
                                            : shares(2048, key_tiles, kKeys, rows, mfma ? 24 : 16);
    }
    p.near = {nullptr, (int32_t)groups, splits};
    p.near_bytes = p.near.splits == 1 ? 0 : rounded((size_t)(slices * groups * p.near.splits) * 64 * D * sizeof(float));

    p.far = {nullptr, 0, 0, p.narrow ? 32 : kKeys};
    p.far_bytes = 0;
    // queries beyond the window of a sink exist where the window is shorter than the sequence
    if (s.sinks == 0 || s.left >= s.k_tokens) return p;
    Far& f = p.far;
    f.groups = (s.sinks + 31) / 32;
    // One workgroup of the narrow kernel runs on a CU: a round of them, or what the groups of 32 keys of
    // the same launch leave of their last round, of at least 8 tiles of 32 queries each.
    const int64_t beside = slices * groups * p.near.splits;
    const int64_t room = p.narrow ? max((int64_t)64, (beside + 255) / 256 * 256 - beside) : 256;
    const int64_t want = max((int64_t)1, room / (slices * f.groups)), most = max(1, s.rows / 256);
    f.chunks = (int)min(min(want, most), (int64_t)32);
    p.far_bytes = rounded((size_t)slices * f.groups * (f.chunks + 1) * 64 * D * sizeof(float));
    return p;
}

template <typename T, int D>
hipError_t launch_bwd(const Shape& s, const void* q_, const void* k_, const void* v_, const void* out_,
                      const float* lse, const void* dout_, void* dq_, void* dk_, void* dv_,
                      void* workspace, hipStream_t stream)
{
    const T *q = (const T*)q_, *k = (const T*)k_, *v = (const T*)v_, *out = (const T*)out_,
            *dout = (const T*)dout_;
    T *dq = (T*)dq_, *dk = (T*)dk_, *dv = (T*)dv_;
    const int64_t slices = (int64_t)s.batch * s.kv_heads;
    float* delta = (float*)workspace;
    float* lse2 = (float*)((char*)workspace + row_bytes(s));
    const bool mfma = window_bwd_mfma_supported(sizeof(T) == 2, D, s);
    Plan plan = plan_of(mfma, (int)sizeof(T), D, s);
    Far& far = plan.far;
    Near& near = plan.near;
    const bool narrow = plan.narrow;
    far.sums = (float*)((char*)workspace + 2 * row_bytes(s));
    near.sums = (float*)((char*)far.sums + plan.far_bytes);

    hipError_t e;
    // Launches of few workgroups of 128 rows: 32 rows to each.  The matrix-core kernels, which take a launch
    // more, are the faster ones from about 256 on, at head dim 128 from 192 (us, backward, narrow | not: head dim
    // 64, 111 workgroups 51 | 79, 235 83 | 111, 264 36 | 28; 128, 150 130 | 167, 208 138 | 106).
    const bool few_rows = slices * (((int64_t)s.rows + 127) / 128) < (mfma && D == 128 ? 192 : 256);
    if (!few_rows && mfma) {
        e = launch_window_dq_mfma(D, s, q, k, v, lse, dout, delta, lse2, dq, stream);
    } else {
        const uint32_t per = few_rows ? 32 : 128, row_tiles = ((uint32_t)s.rows + per - 1) / per;
        const uint32_t q_items = row_tiles * (uint32_t)slices;
        auto kernel = few_rows ? window_dq_kernel<T, D, true> : window_dq_kernel<T, D, false>;
        kernel<<<q_items, 256, 0, stream>>>(q, k, v, out, lse, dout, delta, lse2, dq, s, row_tiles,
                                            q_items);
        e = hipGetLastError();
    }
    if (e != hipSuccess) return e;

    const uint32_t per = narrow ? 32 : kKeys;
    const uint32_t key_tiles = ((uint32_t)s.k_tokens + per - 1) / per;
    const uint32_t k_items = (uint32_t)slices * key_tiles;
    const uint32_t far_items = (uint32_t)slices * (uint32_t)(far.groups * far.chunks);
    const uint32_t narrow_items = far_items + (narrow ? k_items * (uint32_t)near.splits : 0);
    if (narrow_items) {
        window_dkdv_narrow_kernel<T, D><<<narrow_items, 64 * narrow_waves<T, D>(), 0, stream>>>(
            q, k, v, dout, delta, lse2, dk, dv, s, far, near, key_tiles, far_items, k_items);
        if ((e = hipGetLastError()) != hipSuccess) return e;
    }
    if (!narrow) {
        if (mfma) {
            e = launch_window_dkdv_mfma(D, s, q, k, v, dout, delta, lse2, dk, dv, far, near, stream);
        } else {
            window_dkdv_kernel<T, D><<<k_items * (uint32_t)near.splits, 256, 0, stream>>>(
                q, k, v, dout, delta, lse2, dk, dv, s, far, near, key_tiles, k_items);
            e = hipGetLastError();
        }
        if (e != hipSuccess) return e;
    }
    const int groups = near.splits > 1 ? near.groups : narrow ? far.groups : 0;
    if (groups == 0) return hipSuccess;
    const int64_t quads = slices * groups * (16 * D);
    window_keys_kernel<T, D><<<(unsigned)((quads + 255) / 256), 256, 0, stream>>>(dk, dv, s, far, near,
                                                                                 groups, quads);
    return hipGetLastError();
}

}  // namespace win

size_t window_bwd_workspace(bool is_bf16, int D, const win::Shape& s)
{
    // (without strides, on which the choice of kernels depends: enough for either)
    size_t most = 0;
    for (const bool mfma : {false, true}) {
        if (mfma && !(is_bf16 && D >= 64)) continue;
        const win::Plan p = win::plan_of(mfma, is_bf16 ? 2 : 4, D, s);
        most = std::max(most, p.far_bytes + p.near_bytes);
    }
    return 2 * win::row_bytes(s) + most;
}

hipError_t launch_window_bwd(bool is_bf16, int D, const win::Shape& s, const void* q, const void* k,
                             const void* v, const void* out, const float* lse, const void* dout,
                             void* dq, void* dk, void* dv, void* workspace, hipStream_t stream)
{
    using namespace win;
#define BSA_WINDOW_BWD(T, D_) \
    launch_bwd<T, D_>(s, q, k, v, out, lse, dout, dq, dk, dv, workspace, stream)
    if (is_bf16)
        return D == 32   ? BSA_WINDOW_BWD(uint16_t, 32)
               : D == 64 ? BSA_WINDOW_BWD(uint16_t, 64)
                         : BSA_WINDOW_BWD(uint16_t, 128);
    return D == 32   ? BSA_WINDOW_BWD(float, 32)
           : D == 64 ? BSA_WINDOW_BWD(float, 64)
                     : BSA_WINDOW_BWD(float, 128);
#undef BSA_WINDOW_BWD
}

}  // namespace bsa
