// Rotation of query and key heads by their positions, and the root-mean-square norm of
// each head with the rotation in the same pass; both with their gradients.
//
//   forward   z = w x r,  r = (mean(x^2) + eps)^(-1/2),  y = R z   (rotation alone: z = x)
//   backward  dz = R^T dy,  dw = sum over rows of dz x r,  dn = w dz,
//             dx = r (dn - x r mean(dn x r))
// R turns channel pairs by position * frequency and leaves the channels behind rotary_dim.
//
// A row (one head of one token) is read once and written once, so memory bandwidth bounds
// all of it.  A row belongs to P neighbouring lanes, each with two chunks of V channels
// that hold whole pairs (channels c and c + half, or 2V consecutive ones); a wavefront takes
// 64 / P tokens and walks their heads, so that the cosines and sines of a token, the one
// costly piece of arithmetic, are made once for all of its heads and stay in registers.
// They are made in the kernel instead of read from a table: a frequency is held as turns
// per position in units of 2^-64, and the low 64 bits of its product with a 32-bit position
// are the turn's fraction; its upper 32 bits give the angle to 2^-31 turns, 3e-9 radians, for
// any position (frequencies up to 1 radian), where an angle in fp32 is off by 0.03 at position 10^6.
#include "bsa_heads.h"

#include <math.h>

#include "bsa_device.h"
#include "bsa_launch.h"

namespace bsa {

namespace heads {

typedef __attribute__((ext_vector_type(4))) int32_t i32x4;
typedef __attribute__((ext_vector_type(2))) int32_t i32x2;

// One of q, k, v: what a call reads (x; g: the gradient of the result) and writes.
struct Segment {
    const void *x, *g;
    void* y;
    const float* weight;
    mosaic_bsa_strides xs, gs, ys;
    int32_t heads;
    int32_t to_rows;          // y's rows are looked up
};

// Where new tokens of a cache in pages go, and which tokens there are: q_lens and k_lens by sequence.
struct Pages {
    const int32_t *q_lens, *k_lens, *table, *prefix_len;
    int32_t pages, page_shift, table_pages, prefix_tokens;
};

struct Args {
    Segment seg[3];           // q, k, v (v: copied)
    const int32_t* positions;
    const int32_t* rows;
    float* partial;           // backward: [workgroups][2][D]
    int32_t tokens, all_tokens, position_batch, axes, cache_tokens;
    int32_t rotary_dim, axis_dim;
    int32_t rotated_units, units;      // of a row: lanes with pairs, lanes with channels
    int32_t all_heads, head_chunk, chunks;
    float eps, magnitude, sin_magnitude;     // (the transpose turns the other way)
    uint64_t turns[MOSAIC_BSA_MAX_PAIRS];
    Pages paged;
};

// V channels of a row, as they lie in memory (32-bit words; V = 1 in bf16: one in a word).
template <typename T, int V>
struct Chunk {
    static constexpr int WORDS = sizeof(T) * V < 4 ? 1 : (int)sizeof(T) * V / 4;
    uint32_t w[WORDS];
    __device__ __forceinline__ void load(const T* p)
    {
        if constexpr (WORDS == 4) {
            const i32x4 r = *(const i32x4*)p;
#pragma unroll
            for (int i = 0; i < 4; ++i) w[i] = (uint32_t)r[i];
        } else if constexpr (WORDS == 2) {
            const i32x2 r = *(const i32x2*)p;
            w[0] = (uint32_t)r[0];
            w[1] = (uint32_t)r[1];
        } else if constexpr (sizeof(T) * V == 4) {
            w[0] = *(const uint32_t*)p;
        } else {
            w[0] = *p;
        }
    }
    __device__ __forceinline__ float value(int i) const
    {
        if constexpr (sizeof(T) == 4) return __uint_as_float(w[i]);
        else return __uint_as_float((i & 1) ? w[i / 2] & 0xffff0000u : w[i / 2] << 16);
    }
};
// A lane's two chunks of a row; zeros where it has none.
template <typename T, int V>
struct Piece {
    Chunk<T, V> a, b;
    __device__ __forceinline__ void load(const T* p, int ch_a, int ch_b, bool has_a, bool has_b)
    {
#pragma unroll
        for (int i = 0; i < Chunk<T, V>::WORDS; ++i) a.w[i] = b.w[i] = 0u;
        if (has_a) a.load(p + ch_a);
        if (has_b) b.load(p + ch_b);
    }
    __device__ __forceinline__ void values(float (&e)[2 * V]) const
    {
#pragma unroll
        for (int i = 0; i < V; ++i) {
            e[i] = a.value(i);
            e[V + i] = b.value(i);
        }
    }
};

template <typename T, int V>
__device__ __forceinline__ void store_chunk(T* p, const float (&e)[2 * V], int at)
{
    if constexpr (sizeof(T) == 4) {
        if constexpr (V == 4) *(float4*)p = make_float4(e[at], e[at + 1], e[at + 2], e[at + 3]);
        else if constexpr (V == 2) *(float2*)p = make_float2(e[at], e[at + 1]);
        else *p = e[at];
    } else {
        if constexpr (V == 8)
            *(uint4*)p = make_uint4(pack_bf16(e[at], e[at + 1]), pack_bf16(e[at + 2], e[at + 3]),
                                    pack_bf16(e[at + 4], e[at + 5]), pack_bf16(e[at + 6], e[at + 7]));
        else if constexpr (V == 4)
            *(uint2*)p = make_uint2(pack_bf16(e[at], e[at + 1]), pack_bf16(e[at + 2], e[at + 3]));
        else if constexpr (V == 2) *(uint32_t*)p = pack_bf16(e[at], e[at + 1]);
        else *p = (uint16_t)pack_bf16(e[at], 0.0f);
    }
}

// Cosine and sine of u / 2^32 turns.  The nearest quarter turn is taken off, which leaves
// |x| <= pi / 4, where the Taylor polynomials of degree 9 and 10 are off by 2e-9.
__device__ __forceinline__ void cos_sin(uint32_t u, float& c, float& s)
{
    const uint32_t quarter = (u + 0x20000000u) >> 30;
    const float x = (float)(int32_t)(u - (quarter << 30)) * 1.4629180792671596e-9f;  // 2 pi / 2^32
    const float y = x * x;
    const float sp = x * fmaf(y, fmaf(y, fmaf(y, fmaf(y, 2.7557319e-6f, -1.9841270e-4f),
                                              8.3333333e-3f), -0.16666667f), 1.0f);
    const float cp = fmaf(y, fmaf(y, fmaf(y, fmaf(y, fmaf(y, -2.7557319e-7f, 2.4801587e-5f),
                                                  -1.3888889e-3f), 4.1666667e-2f), -0.5f), 1.0f);
    const float a = quarter & 1 ? sp : cp, b = quarter & 1 ? cp : sp;
    c = (quarter + 1) & 2 ? -a : a;
    s = quarter & 2 ? -b : b;
}

enum { kRotate, kNorm, kNormGrad };

template <int CTRL>
__device__ __forceinline__ float add_lane(float x)
{
    return x + __uint_as_float((uint32_t)__builtin_amdgcn_update_dpp(0, (int)__float_as_uint(x), CTRL, 0xf,
                                                                     0xf, true));
}
// Sum over the P (a power of two) lanes of a row: neighbours, pairs, then mirrored halves of 8 and 16
// lanes, which data-parallel moves reach without LDS.
__device__ __forceinline__ float row_sum(float x, int P)
{
    if (P > 1) x = add_lane<0xb1>(x);                  // lanes 1 0 3 2
    if (P > 2) x = add_lane<0x4e>(x);                  // lanes 2 3 0 1
    if (P > 4) x = add_lane<0x141>(x);                 // mirrored in 8
    if (P > 8) x = add_lane<0x140>(x);                 // mirrored in 16
    if (P > 16) x += __shfl_xor(x, 16);
    if (P > 32) x += __shfl_xor(x, 32);
    return x;
}

// PAGED (kRotate, kNorm): a token is the q_lens[b] - n-th from the end of its sequence, which gives its
// position, where none are given, and the page and row that keys and values go to.
template <typename T, int V, bool PAIRS, int MODE, bool PAGED>
__global__ __launch_bounds__(256, 3) void heads_kernel(const Args a, const int D, const int P)
{
    constexpr int E = 2 * V;
    constexpr int U = MODE == kNormGrad ? 1 : 2;     // heads at a time
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int unit = lane & (P - 1), slot = lane / P, per_wave = 64 / P;
    const bool active = unit < a.units, rotated = unit < a.rotated_units;

    // this lane's two chunks and its first pair
    int ch_a, ch_b, axis = 0, pair0 = 0;
    if (rotated) {
        const int per_axis = a.axis_dim / E;
        axis = unit / per_axis;
        pair0 = (unit - axis * per_axis) * V;
        ch_a = axis * a.axis_dim + (PAIRS ? 2 * pair0 : pair0);
        ch_b = ch_a + (PAIRS ? V : a.axis_dim / 2);
    } else {
        ch_a = a.rotary_dim + (unit - a.rotated_units) * E;
        ch_b = ch_a + V;
    }
    const bool has_b = active && ch_b < D;

    float wsum[2][MODE == kNormGrad ? E : 1];
    if constexpr (MODE == kNormGrad)
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int i = 0; i < E; ++i) wsum[t][i] = 0.0f;

    const int per_group = 4 * per_wave;
    const uint32_t groups = ((uint32_t)a.all_tokens + per_group - 1) / per_group;
    const uint32_t items = groups * (uint32_t)a.chunks;
    for (uint32_t item = blockIdx.x; item < items; item += gridDim.x) {
        const uint32_t group = item / (uint32_t)a.chunks;
        const int head0 = (int)(item - group * a.chunks) * a.head_chunk;
        const int head1 = min(a.all_heads, head0 + a.head_chunk);
        const uint32_t tok = group * per_group + wave * per_wave + slot;
        bool here = active && tok < (uint32_t)a.all_tokens;
        const uint32_t tk = tok < (uint32_t)a.all_tokens ? tok : 0u;
        const int b = (int)(tk / (uint32_t)a.tokens), n = (int)(tk - (uint32_t)b * a.tokens);
        int place = 0, page = -1, prefix = 0;         // PAGED: index among the sequence's own tokens; its page
        if constexpr (PAGED) {
            const Pages& pg = a.paged;
            const int ql = pg.q_lens ? min(max(pg.q_lens[b], 0), a.tokens) : a.tokens;
            const int kl = min(max(pg.k_lens[b], 0), pg.table_pages << pg.page_shift);
            if (pg.prefix_len) prefix = min(max(*pg.prefix_len, 0), pg.prefix_tokens);
            else prefix = pg.prefix_tokens;
            place = kl - ql + n;
            here = here && n < ql;
            if (here && place >= 0)
                page = pg.table[(int64_t)b * pg.table_pages + (place >> pg.page_shift)];
        }

        float cs[V], sn[V];
#pragma unroll
        for (int i = 0; i < V; ++i) { cs[i] = 1.0f; sn[i] = 0.0f; }
        if (rotated) {
            const int32_t pos = a.positions
                                    ? a.positions[(int64_t)b * a.position_batch + (int64_t)n * a.axes + axis]
                                    : PAGED ? prefix + place : n;
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const uint64_t turn = (uint64_t)(int64_t)pos * a.turns[pair0 + i];
                cos_sin((uint32_t)(turn >> 32), cs[i], sn[i]);
                cs[i] *= a.magnitude;
                sn[i] *= a.sin_magnitude;
            }
        }

        int seg0 = 0;
        for (int si = 0; si < 3; ++si) {
            const Segment& sg = a.seg[si];
            const int from = max(head0 - seg0, 0), to = min(head1 - seg0, sg.heads);
            seg0 += sg.heads;
            if (from >= to) continue;
            const bool copy = si == 2;
            bool write = here;
            int64_t row = n;
            int64_t block = b;
            if constexpr (PAGED) {
                if (si > 0) {
                    row = place & ((1 << a.paged.page_shift) - 1);
                    block = page;
                    write = here && (uint32_t)page < (uint32_t)a.paged.pages;
                }
            } else if (sg.to_rows) {
                row = a.rows[tk];
                write = here && row >= 0 && row < a.cache_tokens;
            }
            const T* x = (const T*)sg.x + (int64_t)b * sg.xs.batch + (int64_t)n * sg.xs.token;
            const T* g = (const T*)sg.g + (int64_t)b * sg.gs.batch + (int64_t)n * sg.gs.token;
            T* y = (T*)sg.y + block * sg.ys.batch + row * sg.ys.token;
            float w[MODE >= kNorm ? E : 1];
            if constexpr (MODE >= kNorm) {
                if (!copy) {
#pragma unroll
                    for (int i = 0; i < V; ++i) {
                        w[i] = active ? sg.weight[ch_a + i] : 0.0f;
                        w[V + i] = has_b ? sg.weight[ch_b + i] : 0.0f;
                    }
                }
            }
            // The rows of the next U heads are asked for before these are worked on.
            Piece<T, V> xn[U], gn[MODE == kNormGrad ? U : 1];
            auto ask = [&](int h) {
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    const bool there = here && h + u < to;
                    xn[u].load(x + (int64_t)(h + u) * sg.xs.head, ch_a, ch_b, there, there && has_b);
                    if constexpr (MODE == kNormGrad)
                        gn[u].load(g + (int64_t)(h + u) * sg.gs.head, ch_a, ch_b, there, there && has_b);
                }
            };
            ask(from);
            for (int h = from; h < to; h += U) {
                float e[U][E], d[MODE == kNormGrad ? U : 1][MODE == kNormGrad ? E : 1];
                Piece<T, V> xc[U], gc[MODE == kNormGrad ? U : 1];
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    xc[u] = xn[u];
                    if constexpr (MODE == kNormGrad) gc[u] = gn[u];
                }
                if (h + U < to) ask(h + U);
                auto turn = [&](float (&z)[E]) {
#pragma unroll
                    for (int i = 0; i < V; ++i) {
                        const int p0 = PAIRS ? 2 * i : i, p1 = PAIRS ? 2 * i + 1 : V + i;
                        const float z0 = z[p0], z1 = z[p1];
                        z[p0] = fmaf(z0, cs[i], -(z1 * sn[i]));
                        z[p1] = fmaf(z1, cs[i], z0 * sn[i]);
                    }
                };
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    if (h + u >= to) break;
                    xc[u].values(e[u]);
                    if constexpr (MODE == kNormGrad) gc[u].values(d[u]);
                    if constexpr (MODE == kRotate) {
                        if (!copy) turn(e[u]);
                    } else {
                        if (!copy) {
                            float sq = 0.0f;
#pragma unroll
                            for (int i = 0; i < E; ++i) sq = fmaf(e[u][i], e[u][i], sq);
                            sq = row_sum(sq, P);
                            float r = 1.0f / sqrtf(sq * (1.0f / (float)D) + a.eps);
                            // (lanes without a row hold zeros, and without an epsilon r is infinite
                            // there: the weights' sums take all lanes)
                            if (MODE == kNormGrad && !here) r = 0.0f;
                            if constexpr (MODE == kNorm) {
#pragma unroll
                                for (int i = 0; i < E; ++i) e[u][i] *= r * w[i];
                                turn(e[u]);
                            } else {
                                turn(d[u]);
                                float dot = 0.0f;
#pragma unroll
                                for (int i = 0; i < E; ++i) {
                                    e[u][i] *= r;
                                    wsum[si & 1][i] = fmaf(d[u][i], e[u][i], wsum[si & 1][i]);
                                    d[u][i] *= w[i];
                                    dot = fmaf(d[u][i], e[u][i], dot);
                                }
                                dot = row_sum(dot, P) * (1.0f / (float)D);
#pragma unroll
                                for (int i = 0; i < E; ++i)
                                    e[u][i] = r * fmaf(-dot, e[u][i], d[u][i]);
                            }
                        }
                    }
                    T* p = y + (int64_t)(h + u) * sg.ys.head;
                    if (write) store_chunk<T, V>(p + ch_a, e[u], 0);
                    if (write && has_b) store_chunk<T, V>(p + ch_b, e[u], V);
                }
            }
        }
    }

    if constexpr (MODE == kNormGrad) {
        // rows of the wavefront, then the wavefronts, in a fixed order
        __shared__ float sums[4][2][128];
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int i = 0; i < E; ++i) {
                float x = wsum[t][i];
                for (int o = P; o < 64; o <<= 1) x += __shfl_xor(x, o);
                if (slot == 0 && active && (i < V || has_b))
                    sums[wave][t][i < V ? ch_a + i : ch_b + i - V] = x;
            }
        __syncthreads();
        if ((int)threadIdx.x < 2 * D) {
            const int t = threadIdx.x / D, c = threadIdx.x - t * D;
            a.partial[((int64_t)blockIdx.x * 2 + t) * D + c] =
                (sums[0][t][c] + sums[1][t][c]) + (sums[2][t][c] + sums[3][t][c]);
        }
    }
}

// dw = sum of the workgroups' parts in a fixed order, in 64 bits.  One workgroup per four columns of
// the [workgroups][2 D] parts.
__global__ __launch_bounds__(256) void weight_grad_kernel(const float* __restrict__ partial,
                                                          int workgroups, int D, float* dqw,
                                                          float* dkw)
{
    __shared__ double sums[256][4];
    const int col = blockIdx.x * 4, at = threadIdx.x;
    double s[4] = {0.0, 0.0, 0.0, 0.0};
    for (int w = at; w < workgroups; w += 256) {
        const float4 x = *(const float4*)(partial + (int64_t)w * 2 * D + col);
        s[0] += (double)x.x; s[1] += (double)x.y; s[2] += (double)x.z; s[3] += (double)x.w;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) sums[at][i] = s[i];
    for (int o = 128; o > 0; o >>= 1) {
        __syncthreads();
        if (at < o)
#pragma unroll
            for (int i = 0; i < 4; ++i) sums[at][i] += sums[at + o][i];
    }
    if (at == 0) {
        float* to = col < D ? dqw + col : dkw ? dkw + (col - D) : nullptr;
        if (to)
            for (int i = 0; i < 4; ++i) to[i] = (float)sums[0][i];
    }
}

// Workgroups whose parts the backward of the norm leaves: three to a CU, as many as run at once with
// the registers of its widest form (1,024: a round and a third), of which three wavefronts per SIMD leave 168:
// 12 (pairs) and 27 (halves) values of the 8-channel bf16 form spill.  4 x 28,800 tokens, 16 + 4 heads, head dim 128:
// 401 us, 4.4 TB/s.
constexpr int kGradWorkgroups = 768;

template <typename T, int V, bool PAIRS>
hipError_t launch_mode(const Args& a, int mode, int D, int P, unsigned grid, hipStream_t stream)
{
#define BSA_HEADS(MODE, PAGED) heads_kernel<T, V, PAIRS, MODE, PAGED><<<grid, 256, 0, stream>>>(a, D, P)
    if (a.paged.k_lens) {
        if (mode == kRotate) BSA_HEADS(kRotate, true);
        else BSA_HEADS(kNorm, true);
    } else {
        switch (mode) {
        case kRotate: BSA_HEADS(kRotate, false); break;
        case kNorm: BSA_HEADS(kNorm, false); break;
        default: BSA_HEADS(kNormGrad, false); break;
        }
    }
#undef BSA_HEADS
    return hipGetLastError();
}

template <typename T, int V>
hipError_t launch_layout(bool pairs, const Args& a, int mode, int D, int P, unsigned grid,
                         hipStream_t stream)
{
    return pairs ? launch_mode<T, V, true>(a, mode, D, P, grid, stream)
                 : launch_mode<T, V, false>(a, mode, D, P, grid, stream);
}

struct Checked {
    int D, kv_heads;
    bool is_bf16;
};

int check_params(const mosaic_bsa_heads_params* p, Checked* c)
{
    if (!p) return MOSAIC_BSA_ERR_NULL;
    if (p->batch <= 0 || p->tokens <= 0 || p->heads <= 0 || p->kv_heads < 0 ||
        p->cache_tokens < 0 || p->position_batch < 0 || p->heads > (1 << 20) ||
        p->kv_heads > (1 << 20) || (int64_t)p->batch * p->tokens > (int64_t)1 << 30)
        return MOSAIC_BSA_ERR_SHAPE;
    if (p->head_dim != 32 && p->head_dim != 64 && p->head_dim != 128) return MOSAIC_BSA_ERR_HEAD_DIM;
    if (p->dtype != MOSAIC_BSA_F32 && p->dtype != MOSAIC_BSA_BF16) return MOSAIC_BSA_ERR_DTYPE;
    // (also refuses NaN)
    if (!(p->norm_eps >= 0.0f && p->norm_eps < INFINITY)) return MOSAIC_BSA_ERR_SHAPE;
    c->D = p->head_dim;
    c->kv_heads = p->kv_heads == 0 ? p->heads : p->kv_heads;
    c->is_bf16 = p->dtype == MOSAIC_BSA_BF16;
    return MOSAIC_BSA_OK;
}

int check_rotation(const mosaic_bsa_rotation* r, const Checked& c, const int32_t* positions)
{
    if (!r) return MOSAIC_BSA_ERR_NULL;
    if ((r->axes != 1 && r->axes != 2) || r->rotary_dim < 0 || r->rotary_dim > c.D ||
        r->rotary_dim % (2 * r->axes) ||
        (r->layout != MOSAIC_BSA_ROTATE_HALVES && r->layout != MOSAIC_BSA_ROTATE_PAIRS) ||
        !(fabsf(r->magnitude) < INFINITY))
        return MOSAIC_BSA_ERR_ROTATION;
    // grid positions have no default
    if (r->axes == 2 && !positions && r->rotary_dim > 0) return MOSAIC_BSA_ERR_NULL;
    return MOSAIC_BSA_OK;
}

// Fills the rest of `a` (segments, positions, rows, partial, eps are there), checks alignment
// and launches.  grid_limit: most workgroups; *used: how many there are.
int launch(Args& a, const mosaic_bsa_heads_params* p, const Checked& c,
           const mosaic_bsa_rotation* r, int mode, bool transpose, int64_t grid_limit,
           unsigned* used, hipStream_t stream)
{
    const int esz = c.is_bf16 ? 2 : 4;
    const int d = r->rotary_dim / r->axes;
    // The widest chunks (16 bytes at most) that hold whole pairs and that every base and
    // stride is a multiple of.
    int V = 16 / esz;
    auto fits = [&](const void* ptr, const mosaic_bsa_strides& s) {
        return !ptr || ((uintptr_t)ptr % (V * esz) == 0 && s.batch % V == 0 && s.head % V == 0 &&
                        s.token % V == 0);
    };
    for (; V > 1; V >>= 1) {
        bool ok = d % (2 * V) == 0 && (c.D - r->rotary_dim) % V == 0;
        for (const Segment& s : a.seg)
            if (s.heads) ok = ok && fits(s.x, s.xs) && fits(s.g, s.gs) && fits(s.y, s.ys);
        if (ok) break;
    }
    a.tokens = p->tokens;
    a.all_tokens = p->batch * p->tokens;
    a.position_batch = p->position_batch;
    a.axes = r->axes;
    a.cache_tokens = p->cache_tokens;
    a.rotary_dim = r->rotary_dim;
    a.axis_dim = d;
    a.rotated_units = r->rotary_dim / (2 * V);
    a.units = a.rotated_units + (c.D - r->rotary_dim + 2 * V - 1) / (2 * V);
    a.magnitude = r->magnitude;
    a.sin_magnitude = transpose ? -r->magnitude : r->magnitude;
    for (int i = 0; i < d / 2; ++i) a.turns[i] = r->turns[i];
    int P = 1;
    while (P < a.units) P <<= 1;
    a.all_heads = a.seg[0].heads + a.seg[1].heads + a.seg[2].heads;
    // Heads of a token stay together, so that its angles are made once: all of them while that
    // gives 8,192 workgroups, else 8 or more (a launch of one round of workgroups and a few ends with
    // those few alone on the chip), and fewer where less than four wavefronts per SIMD would be left.
    const int64_t groups = ((int64_t)a.all_tokens + 4 * (64 / P) - 1) / (4 * (64 / P));
    const int64_t even = (8192 + groups - 1) / groups, most = (a.all_heads + 7) / 8;
    int64_t chunks = even < most ? even : most;
    if (groups * chunks < 1024) chunks = (1024 + groups - 1) / groups;
    if (chunks > a.all_heads) chunks = a.all_heads;
    a.head_chunk = (int)((a.all_heads + chunks - 1) / chunks);
    a.chunks = (a.all_heads + a.head_chunk - 1) / a.head_chunk;
    const int64_t items = groups * a.chunks;
    if (items >= (int64_t)1 << 31) return MOSAIC_BSA_ERR_SHAPE;
    const unsigned grid = (unsigned)(items < grid_limit ? items : grid_limit);
    if (used) *used = grid;
    const bool pairs = r->layout == MOSAIC_BSA_ROTATE_PAIRS;
    hipError_t e;
    if (c.is_bf16)
        e = V == 8   ? launch_layout<uint16_t, 8>(pairs, a, mode, c.D, P, grid, stream)
            : V == 4 ? launch_layout<uint16_t, 4>(pairs, a, mode, c.D, P, grid, stream)
            : V == 2 ? launch_layout<uint16_t, 2>(pairs, a, mode, c.D, P, grid, stream)
                     : launch_layout<uint16_t, 1>(pairs, a, mode, c.D, P, grid, stream);
    else
        e = V == 4   ? launch_layout<float, 4>(pairs, a, mode, c.D, P, grid, stream)
            : V == 2 ? launch_layout<float, 2>(pairs, a, mode, c.D, P, grid, stream)
                     : launch_layout<float, 1>(pairs, a, mode, c.D, P, grid, stream);
    return e == hipSuccess ? MOSAIC_BSA_OK : MOSAIC_BSA_ERR_LAUNCH;
}

constexpr int64_t kMostWorkgroups = 1 << 20;

bool unaligned(const void* p, int to) { return ((uintptr_t)p % to) != 0; }

// One tensor pair of a call: null both or neither, element alignment, strides.
int check_pair(const void* in, const void* out, bool required, const mosaic_bsa_strides& is,
               const mosaic_bsa_strides& os, int64_t batch, int64_t heads, int64_t tokens,
               int64_t out_tokens, const Checked& c)
{
    if (!in != !out || (required && !in)) return MOSAIC_BSA_ERR_NULL;
    if (!in) return MOSAIC_BSA_OK;
    const int esz = c.is_bf16 ? 2 : 4;
    if (unaligned(in, esz) || unaligned(out, esz)) return MOSAIC_BSA_ERR_ALIGN;
    if (bad_strides(is, batch, heads, tokens, c.D, false) ||
        bad_strides(os, batch, heads, out_tokens, c.D, true) ||
        rows_meet(os, batch, heads, out_tokens, c.D))
        return MOSAIC_BSA_ERR_STRIDE;
    return MOSAIC_BSA_OK;
}

int forward(const mosaic_bsa_heads_params* p, const mosaic_bsa_rotation* r,
            const int32_t* positions, const void* q, const void* k, const void* v,
            const float* q_weight, const float* k_weight, const int32_t* rows, void* q_out,
            void* k_out, void* v_out, bool norm, hipStream_t stream)
{
    Checked c;
    if (int rc = check_params(p, &c)) return rc;
    if (int rc = check_rotation(r, c, positions)) return rc;
    if (norm && (!q_weight || (k && !k_weight))) return MOSAIC_BSA_ERR_NULL;
    const int64_t B = p->batch, N = p->tokens, M = rows ? p->cache_tokens : N;
    if (rows && M <= 0) return MOSAIC_BSA_ERR_SHAPE;
    if (int rc = check_pair(q, q_out, true, p->q, p->q_out, B, p->heads, N, N, c)) return rc;
    if (int rc = check_pair(k, k_out, false, p->k, p->k_out, B, c.kv_heads, N, M, c)) return rc;
    if (int rc = check_pair(v, v_out, false, p->v, p->v_out, B, c.kv_heads, N, M, c)) return rc;
    if (unaligned(positions, 4) || unaligned(rows, 4) || unaligned(q_weight, 4) ||
        unaligned(k_weight, 4))
        return MOSAIC_BSA_ERR_ALIGN;
    const int D = c.D;
    Args a = {};
    const mosaic_bsa_strides none = {0, 0, 0};
    a.seg[0] = {q, nullptr, q_out, q_weight, strides_of(p->q, p->heads, N, D), none,
                strides_of(p->q_out, p->heads, N, D), p->heads, 0};
    a.seg[1] = {k, nullptr, k_out, k_weight, strides_of(p->k, c.kv_heads, N, D), none,
                strides_of(p->k_out, c.kv_heads, M, D), k ? c.kv_heads : 0, rows != nullptr};
    a.seg[2] = {v, nullptr, v_out, nullptr, strides_of(p->v, c.kv_heads, N, D), none,
                strides_of(p->v_out, c.kv_heads, M, D), v ? c.kv_heads : 0, rows != nullptr};
    a.positions = positions;
    a.rows = rows;
    a.eps = p->norm_eps;
    return launch(a, p, c, r, norm ? kNorm : kRotate, false, kMostWorkgroups, nullptr, stream);
}

}  // namespace heads

}  // namespace bsa

using namespace bsa;
using namespace bsa::heads;

extern "C" int mosaic_bsa_rotation_init(int32_t rotary_dim, int32_t axes, int32_t layout,
                                        double theta, int32_t scaling, double factor,
                                        double original_tokens, double beta_fast,
                                        double beta_slow, const double* inv_freq,
                                        mosaic_bsa_rotation* out)
{
    if (!out) return MOSAIC_BSA_ERR_NULL;
    if ((axes != 1 && axes != 2) || rotary_dim < 0 || rotary_dim > 2 * MOSAIC_BSA_MAX_PAIRS ||
        rotary_dim % (2 * axes) ||
        (layout != MOSAIC_BSA_ROTATE_HALVES && layout != MOSAIC_BSA_ROTATE_PAIRS))
        return MOSAIC_BSA_ERR_ROTATION;
    const int d = rotary_dim / axes;
    // (64 bits of mantissa: a double's 53 would leave angles at position 2^31 off by 1e-7)
    long double base = theta;
    if (beta_fast == 0.0 && beta_slow == 0.0) { beta_fast = 32.0; beta_slow = 1.0; }
    if (!inv_freq) {
        if (!(theta > 0.0 && theta < INFINITY) || scaling < MOSAIC_BSA_SCALE_NONE ||
            scaling > MOSAIC_BSA_SCALE_RAMP)
            return MOSAIC_BSA_ERR_ROTATION;
        if (scaling != MOSAIC_BSA_SCALE_NONE && !(factor >= 1.0 && factor < INFINITY))
            return MOSAIC_BSA_ERR_ROTATION;
        if (scaling == MOSAIC_BSA_SCALE_RAMP &&
            !(original_tokens > 0.0 && original_tokens < INFINITY && beta_slow > 0.0 &&
              beta_fast > beta_slow && beta_fast < INFINITY))
            return MOSAIC_BSA_ERR_ROTATION;
        // one pair has one frequency, which a change of the base leaves at 1
        if (scaling == MOSAIC_BSA_SCALE_BASE && d > 2) base *= powl(factor, d / (d - 2.0L));
    }
    mosaic_bsa_rotation t = {};
    t.rotary_dim = rotary_dim;
    t.axes = axes;
    t.layout = layout;
    t.magnitude = !inv_freq && scaling == MOSAIC_BSA_SCALE_RAMP ? (float)(0.1 * log(factor) + 1.0)
                                                                : 1.0f;
    const long double two_pi = 6.283185307179586476925286766559L;
    for (int i = 0; i < d / 2; ++i) {
        long double w;
        if (inv_freq) {
            w = inv_freq[i];
            if (!(fabs(inv_freq[i]) < INFINITY)) return MOSAIC_BSA_ERR_ROTATION;
        } else {
            w = powl(base, -2.0L * i / d);
            if (scaling == MOSAIC_BSA_SCALE_LINEAR) w /= factor;
            if (scaling == MOSAIC_BSA_SCALE_RAMP) {
                long double keep = (original_tokens * w / two_pi - beta_slow) /
                                   ((long double)beta_fast - beta_slow);
                keep = keep < 0.0L ? 0.0L : keep > 1.0L ? 1.0L : keep;
                w = keep * w + (1.0L - keep) * w / factor;
            }
        }
        // turns per position modulo 1, in units of 2^-64 (positions are whole numbers)
        long double turn = w / two_pi;
        turn -= floorl(turn);
        const long double units = rintl(ldexpl(turn, 64));
        t.turns[i] = units >= 18446744073709551616.0L ? 0 : (uint64_t)units;
    }
    *out = t;
    return MOSAIC_BSA_OK;
}

extern "C" int mosaic_bsa_rope_fwd(const mosaic_bsa_heads_params* params,
                                   const mosaic_bsa_rotation* rotation, const int32_t* positions,
                                   const void* q, const void* k, const void* v,
                                   const int32_t* rows, void* q_out, void* k_out, void* v_out,
                                   void* hip_stream)
{
    return forward(params, rotation, positions, q, k, v, nullptr, nullptr, rows, q_out, k_out,
                   v_out, false, (hipStream_t)hip_stream);
}

extern "C" int mosaic_bsa_qk_norm_rope_fwd(const mosaic_bsa_heads_params* params,
                                           const mosaic_bsa_rotation* rotation,
                                           const int32_t* positions, const void* q, const void* k,
                                           const void* v, const float* q_weight,
                                           const float* k_weight, const int32_t* rows, void* q_out,
                                           void* k_out, void* v_out, void* hip_stream)
{
    return forward(params, rotation, positions, q, k, v, q_weight, k_weight, rows, q_out, k_out,
                   v_out, true, (hipStream_t)hip_stream);
}

extern "C" int mosaic_bsa_paged_append(const mosaic_bsa_paged_params* params,
                                       const mosaic_bsa_rotation* rotation,
                                       const int32_t* positions, const void* q, const void* k,
                                       const void* v, const float* q_weight, const float* k_weight,
                                       const int32_t* q_lens, const int32_t* k_lens,
                                       const int32_t* page_table, const int32_t* prefix_len,
                                       void* q_out, void* k_pages, void* v_pages, void* hip_stream)
{
    if (!params) return MOSAIC_BSA_ERR_NULL;
    const mosaic_bsa_paged_params& p = *params;
    mosaic_bsa_heads_params h = {};
    h.batch = p.batch;
    h.tokens = p.q_tokens;
    h.heads = p.heads;
    h.kv_heads = p.kv_heads;
    h.head_dim = p.head_dim;
    h.dtype = p.dtype;
    h.position_batch = p.position_batch;
    h.norm_eps = p.norm_eps;
    Checked c;
    if (int rc = check_params(&h, &c)) return rc;
    if (int rc = check_pages(p)) return rc;
    if (int rc = check_rotation(rotation, c, positions)) return rc;
    if (!q || !k || !v || !q_out || !k_pages || !v_pages || !k_lens || !page_table ||
        !q_weight != !k_weight)
        return MOSAIC_BSA_ERR_NULL;
    const int64_t B = p.batch, N = p.q_tokens, T = p.page_tokens;
    const int kv = c.kv_heads, D = c.D;
    if (int rc = check_pair(q, q_out, true, p.q, p.out, B, p.heads, N, N, c)) return rc;
    const struct { const void* x; const mosaic_bsa_strides* s; int64_t n, rows; bool output; } rest[] = {
        {k, &p.k, B, N, false}, {v, &p.v, B, N, false},
        {k_pages, &p.k_pages, p.pages, T, true}, {v_pages, &p.v_pages, p.pages, T, true}};
    for (const auto& r : rest) {
        if (unaligned(r.x, c.is_bf16 ? 2 : 4)) return MOSAIC_BSA_ERR_ALIGN;
        if (bad_strides(*r.s, r.n, kv, r.rows, D, r.output) ||
            (r.output && rows_meet(*r.s, r.n, kv, r.rows, D)))
            return MOSAIC_BSA_ERR_STRIDE;
    }
    if (unaligned(positions, 4) || unaligned(q_weight, 4) || unaligned(k_weight, 4) ||
        unaligned(q_lens, 4) || unaligned(k_lens, 4) || unaligned(page_table, 4) ||
        unaligned(prefix_len, 4))
        return MOSAIC_BSA_ERR_ALIGN;
    Args a = {};
    const mosaic_bsa_strides none = {0, 0, 0};
    a.seg[0] = {q, nullptr, q_out, q_weight, strides_of(p.q, p.heads, N, D), none,
                strides_of(p.out, p.heads, N, D), p.heads, 0};
    a.seg[1] = {k, nullptr, k_pages, k_weight, strides_of(p.k, kv, N, D), none,
                strides_of(p.k_pages, kv, T, D), kv, 0};
    a.seg[2] = {v, nullptr, v_pages, nullptr, strides_of(p.v, kv, N, D), none,
                strides_of(p.v_pages, kv, T, D), kv, 0};
    a.positions = positions;
    a.eps = p.norm_eps;
    a.paged = {q_lens, k_lens, page_table, prefix_len, p.pages, __builtin_ctz((unsigned)p.page_tokens),
               p.table_pages, p.prefix_tokens};
    return launch(a, &h, c, rotation, q_weight ? kNorm : kRotate, false, kMostWorkgroups, nullptr,
                  (hipStream_t)hip_stream);
}

extern "C" int mosaic_bsa_rope_bwd(const mosaic_bsa_heads_params* params,
                                   const mosaic_bsa_rotation* rotation, const int32_t* positions,
                                   const void* dq_out, const void* dk_out, void* dq, void* dk,
                                   void* hip_stream)
{
    Checked c;
    if (int rc = check_params(params, &c)) return rc;
    if (int rc = check_rotation(rotation, c, positions)) return rc;
    const int64_t B = params->batch, N = params->tokens;
    const mosaic_bsa_heads_params& p = *params;
    if (int rc = check_pair(dq_out, dq, true, p.q_out, p.q, B, p.heads, N, N, c)) return rc;
    if (int rc = check_pair(dk_out, dk, false, p.k_out, p.k, B, c.kv_heads, N, N, c)) return rc;
    if (unaligned(positions, 4)) return MOSAIC_BSA_ERR_ALIGN;
    const int D = c.D;
    Args a = {};
    const mosaic_bsa_strides none = {0, 0, 0};
    a.seg[0] = {dq_out, nullptr, dq, nullptr, strides_of(p.q_out, p.heads, N, D), none,
                strides_of(p.q, p.heads, N, D), p.heads, 0};
    a.seg[1] = {dk_out, nullptr, dk, nullptr, strides_of(p.k_out, c.kv_heads, N, D), none,
                strides_of(p.k, c.kv_heads, N, D), dk ? c.kv_heads : 0, 0};
    a.positions = positions;
    return launch(a, params, c, rotation, kRotate, true, kMostWorkgroups, nullptr,
                  (hipStream_t)hip_stream);
}

extern "C" size_t mosaic_bsa_qk_norm_rope_workspace_bytes(const mosaic_bsa_heads_params* params)
{
    Checked c;
    if (check_params(params, &c) != MOSAIC_BSA_OK) return 0;
    return (size_t)kGradWorkgroups * 2 * c.D * sizeof(float);
}

extern "C" int mosaic_bsa_qk_norm_rope_bwd(
    const mosaic_bsa_heads_params* params, const mosaic_bsa_rotation* rotation,
    const int32_t* positions, const void* q, const void* k, const float* q_weight,
    const float* k_weight, const void* dq_out, const void* dk_out,
    const mosaic_bsa_strides* dq_strides, const mosaic_bsa_strides* dk_strides, void* dq, void* dk,
    float* dq_weight, float* dk_weight, void* workspace, size_t workspace_bytes, void* hip_stream)
{
    Checked c;
    if (int rc = check_params(params, &c)) return rc;
    if (int rc = check_rotation(rotation, c, positions)) return rc;
    const mosaic_bsa_heads_params& p = *params;
    const int64_t B = p.batch, N = p.tokens;
    const mosaic_bsa_strides none = {0, 0, 0};
    const mosaic_bsa_strides qs = dq_strides ? *dq_strides : none;
    const mosaic_bsa_strides ks = dk_strides ? *dk_strides : none;
    if (!q || !q_weight || !dq_weight) return MOSAIC_BSA_ERR_NULL;
    if (dk && (!k || !k_weight || !dk_weight)) return MOSAIC_BSA_ERR_NULL;
    if (int rc = check_pair(dq_out, dq, true, p.q_out, qs, B, p.heads, N, N, c)) return rc;
    if (int rc = check_pair(dk_out, dk, false, p.k_out, ks, B, c.kv_heads, N, N, c)) return rc;
    if (bad_strides(p.q, B, p.heads, N, c.D, false) ||
        (dk && bad_strides(p.k, B, c.kv_heads, N, c.D, false)))
        return MOSAIC_BSA_ERR_STRIDE;
    const int esz = c.is_bf16 ? 2 : 4;
    if (unaligned(q, esz) || (dk && unaligned(k, esz)) || unaligned(positions, 4) ||
        unaligned(q_weight, 4) || unaligned(k_weight, 4) || unaligned(dq_weight, 4) ||
        unaligned(dk_weight, 4) || unaligned(workspace, 16))
        return MOSAIC_BSA_ERR_ALIGN;
    if (!workspace || workspace_bytes < mosaic_bsa_qk_norm_rope_workspace_bytes(params))
        return MOSAIC_BSA_ERR_WORKSPACE;
    const int D = c.D;
    Args a = {};
    a.seg[0] = {q, dq_out, dq, q_weight, strides_of(p.q, p.heads, N, D),
                strides_of(p.q_out, p.heads, N, D), strides_of(qs, p.heads, N, D), p.heads, 0};
    a.seg[1] = {dk ? k : nullptr, dk_out, dk, k_weight, strides_of(p.k, c.kv_heads, N, D),
                strides_of(p.k_out, c.kv_heads, N, D), strides_of(ks, c.kv_heads, N, D),
                dk ? c.kv_heads : 0, 0};
    a.positions = positions;
    a.eps = p.norm_eps;
    a.partial = (float*)workspace;
    unsigned used = 0;
    if (int rc = launch(a, params, c, rotation, kNormGrad, true, kGradWorkgroups, &used,
                        (hipStream_t)hip_stream))
        return rc;
    weight_grad_kernel<<<2 * D / 4, 256, 0, (hipStream_t)hip_stream>>>(
        a.partial, (int)used, D, dq_weight, dk ? dk_weight : nullptr);
    return hipGetLastError() == hipSuccess ? MOSAIC_BSA_OK : MOSAIC_BSA_ERR_LAUNCH;
}
