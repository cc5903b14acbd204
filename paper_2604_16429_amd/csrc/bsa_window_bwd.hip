// Windowed attention backward, any shape the entry point takes, on the matrix cores.
//
// With P = exp(scale q.k - lse) recomputed and delta = dO . O for each query,
//   dV_j = sum_i P_ij dO_i    dS_ij = P_ij (dO_i . v_j - delta_i)
//   dQ_i = scale sum_j dS_ij k_j    dK_j = scale sum_i dS_ij q_i
// Three launches: delta and lse in base 2 by row; dQ, which walks the keys of 128 rows as the
// forward does; dK and dV, where a workgroup owns 128 keys (32 to a wavefront, their K and V rows in
// registers) and walks the rows that see them, all heads of the group in one sequence, so that
// every sum has one fixed order and no atomics.
//
// A sink is seen by every later query, the keys behind it by window ones: the tiles that hold
// sinks would be walked for the whole sequence by one workgroup.  Their rows beyond the window
// are cut into chunks with a workgroup each; the parts meet in fp32 in the workspace and are
// added in the order of the chunks by a fourth launch.
#include "bsa_window.h"

#include "bsa_launch.h"

namespace bsa {

namespace win {

constexpr int kKeys = 128;          // keys of a dK/dV workgroup
constexpr float kNoWeight = 3.0e38f;   // lse of a row without keys: its weights are 0

// What the sinks' far rows are cut into.
struct Far {
    int32_t tiles, chunks;          // key tiles that hold sinks (0: no far rows), chunks of each
};

__host__ __device__ inline int64_t part_floats(int D) { return (int64_t)2 * kKeys * D; }

template <typename T, int D>
__global__ __launch_bounds__(256) void window_rows_kernel(const T* __restrict__ out,
                                                          const T* __restrict__ dout,
                                                          const float* __restrict__ lse,
                                                          float* __restrict__ delta,
                                                          float* __restrict__ lse2, const Shape s,
                                                          int64_t all_rows)
{
    constexpr int LANES = D * sizeof(T) / 16, V = 16 / sizeof(T);
    const int part = threadIdx.x % LANES;
    const int64_t step = (int64_t)gridDim.x * (256 / LANES);
    // (the bound is the same for all lanes of a wavefront, which meet in the sums)
    for (int64_t at0 = (int64_t)blockIdx.x * (256 / LANES); at0 < all_rows; at0 += step) {
        const int64_t at = at0 + threadIdx.x / LANES;
        const bool here = at < all_rows;
        const int64_t slice = here ? at / s.rows : 0;
        const int row = here ? (int)(at - slice * s.rows) : 0;
        const int b = (int)(slice / s.kv_heads), a = (int)(slice - (int64_t)b * s.kv_heads);
        const int tok = row / s.group, head = a * s.group + (row - tok * s.group);
        int ql, kl;
        lengths(s, b, ql, kl);
        const bool valid = here && tok < ql;
        float d = 0.0f;
        if (valid) {
            const T* o = out + (int64_t)b * s.out.batch + (int64_t)head * s.out.head +
                         (int64_t)tok * s.out.token + V * part;
            const T* g = dout + (int64_t)b * s.dout.batch + (int64_t)head * s.dout.head +
                         (int64_t)tok * s.dout.token + V * part;
#pragma unroll
            for (int i = 0; i < V; i += 4) {
                const float4 x = load4(o + i), y = load4(g + i);
                d += x.x * y.x + x.y * y.y + x.z * y.z + x.w * y.w;
            }
        }
#pragma unroll
        for (int o = 1; o < LANES; o <<= 1) d += __shfl_xor(d, o);
        if (here && part == 0) {
            const float l =
                valid ? lse[((int64_t)b * s.heads + head) * s.q_tokens + tok] : -INFINITY;
            delta[at] = d;
            lse2[at] = l == -INFINITY ? kNoWeight : l * kLog2e;
        }
    }
}

template <typename T, int D>
__global__ __launch_bounds__(256) void window_dq_kernel(
    const T* __restrict__ q, const T* __restrict__ k, const T* __restrict__ v,
    const T* __restrict__ dout, const float* __restrict__ delta, const float* __restrict__ lse2,
    T* __restrict__ dq, const Shape s, uint32_t row_tiles, uint32_t items)
{
    constexpr int KT = sizeof(T) == 2 ? 64 : 32;
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
    const int p0 = kl - ql;

    const int row = row0 + 32 * wave + l32;
    const int tok = row / s.group, head = a * s.group + (row - tok * s.group);
    const bool exists = row < s.rows, valid = exists && tok < ql;
    const Sight see = sight(s, p0 + tok, kl, valid);

    const int t_first = row0 / s.group, t_last = min((row0 + 127) / s.group, ql - 1);
    KeyList keys = {};
    if (t_first <= t_last) keys = key_list(s, p0 + t_first, p0 + t_last, kl);
    const int w_first = (row0 + 32 * wave) / s.group, w_end = (row0 + 32 * wave + 31) / s.group;
    const int w_last = min(w_end, ql - 1);
    const int w_lo = p0 + w_first - s.left, w_hi = min(kl - 1, p0 + w_last + s.right);
    const int all_lo = p0 + w_end - s.left, all_hi = min(kl - 1, p0 + w_first + s.right);
    const bool all_valid = w_end < ql && row0 + 32 * wave + 31 < s.rows;

    const T* kb = k + (int64_t)b * s.k.batch + (int64_t)a * s.k.head;
    const T* vb = v + (int64_t)b * s.v.batch + (int64_t)a * s.v.head;

    Frag qf[KS], gf[KS];
    float neg_l2 = -kNoWeight, neg_delta = 0.0f;
    {
        const T* p = q + (int64_t)b * s.q.batch + (int64_t)head * s.q.head + (int64_t)tok * s.q.token;
        const T* g = dout + (int64_t)b * s.dout.batch + (int64_t)head * s.dout.head +
                     (int64_t)tok * s.dout.token;
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
            qf[ks] = valid ? M::load(p + 16 * ks + 8 * half) : Frag{};
            gf[ks] = valid ? M::load(g + 16 * ks + 8 * half) : Frag{};
        }
        if (valid) {
            neg_l2 = -lse2[(int64_t)slice * s.rows + row];
            neg_delta = -delta[(int64_t)slice * s.rows + row];
        }
    }
    const float c2 = s.scale * kLog2e;
    f32x16 acc[DT];
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) acc[dt] = splat(0.0f);

    Tl kt, vt;
    auto fetch = [&](int slot0) {
        kt.fetch(tid, [&](int r) -> const T* {
            const int slot = slot0 + r;
            return slot < keys.count ? kb + (int64_t)keys.token(slot) * s.k.token : nullptr;
        });
        vt.fetch(tid, [&](int r) -> const T* {
            const int slot = slot0 + r;
            return slot < keys.count ? vb + (int64_t)keys.token(slot) * s.v.token : nullptr;
        });
    };
    if (keys.count > 0) fetch(0);
    for (int slot0 = 0; slot0 < keys.count; slot0 += KT) {
        __syncthreads();
        kt.put(k_lds, tid);
        vt.put(v_lds, tid);
        __syncthreads();
        if (slot0 + KT < keys.count) fetch(slot0 + KT);
#pragma unroll
        for (int hh = 0; hh < KT / 32; ++hh) {
            const int s0 = slot0 + 32 * hh, j0 = s0 - keys.sinks + keys.lo;
            const bool plain = s0 >= keys.sinks;
            if (s0 >= keys.count || (plain && (j0 > w_hi || (j0 + 31 < w_lo && j0 >= s.sinks))))
                continue;
            const bool full = plain && all_valid && j0 >= all_lo && j0 + 31 <= all_hi;
            f32x16 st = splat(0.0f), dp = splat(neg_delta);
#pragma unroll
            for (int ks = 0; ks < KS; ++ks) {
                st = M::mul(Tl::row_frag(k_lds, 32 * hh, ks, lane), qf[ks], st);
                dp = M::mul(Tl::row_frag(v_lds, 32 * hh, ks, lane), gf[ks], dp);
            }
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                float ds = __builtin_amdgcn_exp2f(fmaf(st[r], c2, neg_l2)) * dp[r];
                if (!full) {
                    const int slot = s0 + 8 * (r >> 2) + 4 * half + (r & 3);
                    ds = slot < keys.count && see.sees(s, keys.token(slot)) ? ds : 0.0f;
                }
                st[r] = ds;
            }
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const Frag ds = M::pack(st, h);
#pragma unroll
                for (int dt = 0; dt < DT; ++dt)
                    acc[dt] = M::mul(Tl::trans_frag(k_lds, 32 * hh + 16 * h, dt, lane), ds, acc[dt]);
            }
        }
    }
    if (!exists) return;
    store_lane_row<T, D>(dq + (int64_t)b * s.dq.batch + (int64_t)head * s.dq.head +
                             (int64_t)tok * s.dq.token,
                         acc, s.scale, half);
}

// Per slice: key tiles' rows inside the window, then far.tiles * far.chunks chunks of far rows.
template <typename T, int D>
__global__ __launch_bounds__(256) void window_dkdv_kernel(
    const T* __restrict__ q, const T* __restrict__ k, const T* __restrict__ v,
    const T* __restrict__ dout, const float* __restrict__ delta, const float* __restrict__ lse2,
    T* __restrict__ dk, T* __restrict__ dv, float* __restrict__ parts, const Shape s, const Far far,
    uint32_t key_tiles, uint32_t items)
{
    constexpr int RT = sizeof(T) == 2 ? 64 : 32;        // rows of a tile
    constexpr int KS = D / 16, DT = D / 32;
    using Tl = Tile<T, D, RT>;
    using M = Mma<T>;
    using Frag = typename M::Frag;
    __shared__ __attribute__((aligned(1024))) unsigned char q_lds[Tl::BYTES];
    __shared__ __attribute__((aligned(1024))) unsigned char g_lds[Tl::BYTES];
    __shared__ float l2_s[RT], dl_s[RT];
    __shared__ int pos_s[RT];

    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int l32 = lane & 31, half = lane >> 5;

    const uint32_t per_slice = key_tiles + (uint32_t)(far.tiles * far.chunks);
    const uint32_t item = item_of(blockIdx.x, items);
    const uint32_t slice = item / per_slice, in_slice = item - slice * per_slice;
    const bool is_far = in_slice >= key_tiles;
    const int key_tile = is_far ? (int)(in_slice - key_tiles) / far.chunks : (int)in_slice;
    const int chunk = is_far ? (int)(in_slice - key_tiles) - key_tile * far.chunks : 0;
    const int b = (int)(slice / (uint32_t)s.kv_heads), a = (int)(slice - (uint32_t)b * s.kv_heads);
    int ql, kl;
    lengths(s, b, ql, kl);
    const int p0 = kl - ql;
    const int J = key_tile * kKeys;
    const int jw = J + 32 * wave, j = jw + l32;         // this wavefront's keys, this lane's

    // rows that see the tile: query tokens t_a .. t_b
    int t_a = max(0, J - s.right - p0), t_b = min(ql - 1, J + kKeys - 1 + s.left - p0);
    if (J >= kl) t_b = -1;
    int row_a = t_a * s.group, row_e = (t_b + 1) * s.group;
    if (is_far) {
        t_a = max(t_a, J + kKeys + s.left - p0);
        const int rows = J < kl ? max(0, ql - t_a) * s.group : 0;
        const int per = ((rows + far.chunks - 1) / far.chunks + RT - 1) / RT * RT;
        row_a = t_a * s.group + chunk * per;
        row_e = min(t_a * s.group + rows, row_a + per);
    }

    const T* qb = q + (int64_t)b * s.q.batch + (int64_t)a * s.group * s.q.head;
    const T* gb = dout + (int64_t)b * s.dout.batch + (int64_t)a * s.group * s.dout.head;

    Frag kf[KS], vf[KS];
    {
        const bool here = j < kl;
        const T* kp = k + (int64_t)b * s.k.batch + (int64_t)a * s.k.head + (int64_t)j * s.k.token;
        const T* vp = v + (int64_t)b * s.v.batch + (int64_t)a * s.v.head + (int64_t)j * s.v.token;
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
            kf[ks] = here ? M::load(kp + 16 * ks + 8 * half) : Frag{};
            vf[ks] = here ? M::load(vp + 16 * ks + 8 * half) : Frag{};
        }
    }
    const float c2 = s.scale * kLog2e;
    f32x16 ak[DT], av[DT];
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) ak[dt] = av[dt] = splat(0.0f);

    Tl qt, gt;
    float l2_held = 0.0f, dl_held = 0.0f;
    int pos_held = 0;
    auto fetch = [&](int r0) {
        qt.fetch(tid, [&](int r) -> const T* {
            const int row = r0 + r, tok = row / s.group;
            return row < row_e ? qb + (int64_t)(row - tok * s.group) * s.q.head + (int64_t)tok * s.q.token
                               : nullptr;
        });
        gt.fetch(tid, [&](int r) -> const T* {
            const int row = r0 + r, tok = row / s.group;
            return row < row_e
                       ? gb + (int64_t)(row - tok * s.group) * s.dout.head + (int64_t)tok * s.dout.token
                       : nullptr;
        });
        if (tid < RT) {
            const int row = r0 + tid;
            const bool here = row < row_e;
            l2_held = here ? lse2[(int64_t)slice * s.rows + row] : kNoWeight;
            dl_held = here ? delta[(int64_t)slice * s.rows + row] : 0.0f;
            pos_held = here ? p0 + row / s.group : INT32_MIN;      // (sees nothing)
        }
    };
    if (row_a < row_e) fetch(row_a);
    for (int r0 = row_a; r0 < row_e; r0 += RT) {
        __syncthreads();
        qt.put(q_lds, tid);
        gt.put(g_lds, tid);
        if (tid < RT) { l2_s[tid] = l2_held; dl_s[tid] = dl_held; pos_s[tid] = pos_held; }
        __syncthreads();
        if (r0 + RT < row_e) fetch(r0 + RT);
#pragma unroll
        for (int hh = 0; hh < RT / 32; ++hh) {
            const int ra = r0 + 32 * hh, re = min(ra + 32, row_e);
            if (ra >= re) continue;
            const int pa = p0 + ra / s.group, pb = p0 + (re - 1) / s.group;
            if (jw >= kl || jw > pb + s.right || (jw + 31 < pa - s.left && jw >= s.sinks)) continue;
            const bool full = ra + 32 == re && jw + 31 < kl && jw + 31 <= pa + s.right &&
                              (jw >= pb - s.left || jw + 31 < s.sinks);
            f32x16 st = splat(0.0f), dp;
#pragma unroll
            for (int r4 = 0; r4 < 4; ++r4) {
                const f32x4 x = *(const f32x4*)(dl_s + 32 * hh + 8 * r4 + 4 * half);
#pragma unroll
                for (int e = 0; e < 4; ++e) dp[4 * r4 + e] = -x[e];
            }
#pragma unroll
            for (int ks = 0; ks < KS; ++ks) {
                st = M::mul(Tl::row_frag(q_lds, 32 * hh, ks, lane), kf[ks], st);
                dp = M::mul(Tl::row_frag(g_lds, 32 * hh, ks, lane), vf[ks], dp);
            }
#pragma unroll
            for (int r4 = 0; r4 < 4; ++r4) {
                const f32x4 l = *(const f32x4*)(l2_s + 32 * hh + 8 * r4 + 4 * half);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int r = 4 * r4 + e;
                    float w = __builtin_amdgcn_exp2f(fmaf(st[r], c2, -l[e])), ds = w * dp[r];
                    if (!full) {
                        const int p = pos_s[32 * hh + 8 * r4 + 4 * half + e];
                        const bool seen = j < kl && j <= p + s.right && (j >= p - s.left || j < s.sinks);
                        w = seen ? w : 0.0f;
                        ds = seen ? ds : 0.0f;         // (dp of an unseen key may be anything)
                    }
                    st[r] = w;
                    dp[r] = ds;
                }
            }
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const Frag pw = M::pack(st, h), ds = M::pack(dp, h);
#pragma unroll
                for (int dt = 0; dt < DT; ++dt) {
                    av[dt] = M::mul(Tl::trans_frag(g_lds, 32 * hh + 16 * h, dt, lane), pw, av[dt]);
                    ak[dt] = M::mul(Tl::trans_frag(q_lds, 32 * hh + 16 * h, dt, lane), ds, ak[dt]);
                }
            }
        }
    }

    if (key_tile < far.tiles) {
        // one of the parts that are added up: [chunks + 1][2][keys][D]
        float* p = parts + (((int64_t)slice * far.tiles + key_tile) * (far.chunks + 1) +
                            (is_far ? chunk + 1 : 0)) * part_floats(D) + (32 * wave + l32) * D;
        store_lane_row<float, D>(p, ak, s.scale, half);
        store_lane_row<float, D>(p + kKeys * D, av, 1.0f, half);
    } else if (j < s.k_tokens) {
        store_lane_row<T, D>(dk + (int64_t)b * s.dk.batch + (int64_t)a * s.dk.head +
                                 (int64_t)j * s.dk.token, ak, s.scale, half);
        store_lane_row<T, D>(dv + (int64_t)b * s.dv.batch + (int64_t)a * s.dv.head +
                                 (int64_t)j * s.dv.token, av, 1.0f, half);
    }
}

// The tiles that hold sinks: parts in order of the chunks.  A thread has four channels.
template <typename T, int D>
__global__ __launch_bounds__(256) void window_sinks_kernel(const float* __restrict__ parts,
                                                           T* __restrict__ dk, T* __restrict__ dv,
                                                           const Shape s, const Far far,
                                                           int64_t quads)
{
    const int64_t at = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (at >= quads) return;
    const int c = (int)(at % (D / 4)) * 4;
    int64_t rest = at / (D / 4);
    const int key = (int)(rest % kKeys);
    rest /= kKeys;
    const int is_v = (int)(rest & 1);
    const int64_t tile_at = rest >> 1, slice = tile_at / far.tiles;
    const int j = (int)(tile_at - slice * far.tiles) * kKeys + key;
    if (j >= s.k_tokens) return;
    const float* p = parts + tile_at * (far.chunks + 1) * part_floats(D) +
                     ((int64_t)is_v * kKeys + key) * D + c;
    float4 sum = *(const float4*)p;
    for (int i = 1; i <= far.chunks; ++i) {
        const float4 x = *(const float4*)(p + i * part_floats(D));
        sum.x += x.x; sum.y += x.y; sum.z += x.z; sum.w += x.w;
    }
    const int b = (int)(slice / s.kv_heads), a = (int)(slice - (int64_t)b * s.kv_heads);
    T* y = is_v ? dv + (int64_t)b * s.dv.batch + (int64_t)a * s.dv.head + (int64_t)j * s.dv.token
                : dk + (int64_t)b * s.dk.batch + (int64_t)a * s.dk.head + (int64_t)j * s.dk.token;
    store4(y + c, sum);
}

size_t rounded(size_t x) { return (x + 255) & ~(size_t)255; }

size_t row_bytes(const Shape& s)
{
    return rounded((size_t)s.batch * s.kv_heads * s.rows * sizeof(float));
}

Far far_of(const Shape& s)
{
    Far f = {0, 0};
    // queries beyond the window of a sink exist where the window is shorter than the sequence
    if (s.sinks == 0 || s.left >= s.k_tokens) return f;
    f.tiles = (min(s.sinks, s.k_tokens) + kKeys - 1) / kKeys;
    f.chunks = max(1, min(64, s.rows / 1024));
    return f;
}

size_t parts_bytes(const Shape& s, int D)
{
    const Far f = far_of(s);
    if (f.tiles == 0) return 0;
    return rounded((size_t)s.batch * s.kv_heads * f.tiles * (f.chunks + 1) * part_floats(D) *
                   sizeof(float));
}

template <typename T, int D>
hipError_t launch_bwd(const Shape& s, const void* q, const void* k, const void* v, const void* out,
                      const float* lse, const void* dout, void* dq, void* dk, void* dv,
                      void* workspace, hipStream_t stream)
{
    const int64_t slices = (int64_t)s.batch * s.kv_heads;
    float* delta = (float*)workspace;
    float* lse2 = (float*)((char*)workspace + row_bytes(s));
    float* parts = (float*)((char*)workspace + 2 * row_bytes(s));
    const Far far = far_of(s);

    const int64_t all_rows = slices * s.rows;
    const int rows_per = 256 / (D * (int)sizeof(T) / 16);
    const int64_t row_groups = (all_rows + rows_per - 1) / rows_per;
    window_rows_kernel<T, D><<<(unsigned)min(row_groups, (int64_t)1 << 20), 256, 0, stream>>>(
        (const T*)out, (const T*)dout, lse, delta, lse2, s, all_rows);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;

    const uint32_t row_tiles = ((uint32_t)s.rows + 127) / 128;
    const uint32_t q_items = row_tiles * (uint32_t)slices;
    window_dq_kernel<T, D><<<q_items, 256, 0, stream>>>((const T*)q, (const T*)k, (const T*)v,
                                                       (const T*)dout, delta, lse2, (T*)dq, s,
                                                       row_tiles, q_items);
    if ((e = hipGetLastError()) != hipSuccess) return e;

    const uint32_t key_tiles = ((uint32_t)s.k_tokens + kKeys - 1) / kKeys;
    const uint32_t k_items = (uint32_t)slices * (key_tiles + (uint32_t)(far.tiles * far.chunks));
    window_dkdv_kernel<T, D><<<k_items, 256, 0, stream>>>(
        (const T*)q, (const T*)k, (const T*)v, (const T*)dout, delta, lse2, (T*)dk, (T*)dv, parts, s,
        far, key_tiles, k_items);
    if ((e = hipGetLastError()) != hipSuccess) return e;
    if (far.tiles) {
        const int64_t quads = slices * far.tiles * 2 * kKeys * (D / 4);
        window_sinks_kernel<T, D><<<(unsigned)((quads + 255) / 256), 256, 0, stream>>>(
            parts, (T*)dk, (T*)dv, s, far, quads);
        e = hipGetLastError();
    }
    return e;
}

}  // namespace win

size_t window_bwd_workspace(bool, int D, const win::Shape& s)
{
    return 2 * win::row_bytes(s) + win::parts_bytes(s, D);
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
