// Windowed attention forward for few rows (single tokens, chunks, short sequences): a workgroup owns
// 16 or 32 rows (token, head of the group) of a (batch, key/value head) slice.
//
// K and V are read once and used for a handful of rows, so memory bandwidth bounds it, or, where
// the window is short, latency.  A workgroup has 4 wavefronts (or 8 or 16) that take 32 keys each in turn and
// share nothing until the end: no barrier stands between a wavefront and its next loads, which
// are in flight while it works on the keys before.  Rows fill 16-wide matrix instructions: S^T =
// K Q^T, whose K operand is loaded from memory as the lanes hold it, and O^T += V^T P^T, where V goes
// through LDS of the wavefront's own to be read transposed.  At the end the wavefronts' sums meet in LDS
// in the order of the wavefronts; where the keys are split over workgroups, those write parts.
#include "bsa_window.h"

namespace bsa {

namespace win {

// NR: 16-row tiles.  W: wavefronts.
template <typename T, int D, int NR, int W>
__global__ __launch_bounds__(64 * W) void window_step_kernel(
    const T* __restrict__ q, const T* __restrict__ k, const T* __restrict__ v, T* __restrict__ out,
    float* __restrict__ lse, const Shape s, const Parts parts, uint32_t row_tiles, uint32_t items)
{
    constexpr int KS = D / 32, DT = D / 16, KT = 32;
    constexpr int ROW = D * sizeof(T), CHUNKS = ROW / 16;
    constexpr int V_LOADS = KT * CHUNKS / 64;
    constexpr int ACC_BYTES = NR * 16 * D * 4;
    constexpr int REGION = KT * ROW > ACC_BYTES ? KT * ROW : ACC_BYTES;    // of a wavefront
    using Frag = typename Mma<T>::Frag;
    using M = Mma16<T>;
    __shared__ __attribute__((aligned(1024))) unsigned char lds[W * REGION];
    __shared__ float m_s[W][NR * 16], l_s[W][NR * 16];

    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int l16 = lane & 15, grp = lane >> 4;
    unsigned char* const mine = lds + wave * REGION;

    const int split = (int)(blockIdx.x % (uint32_t)parts.splits);
    uint32_t slice;
    int tile_at;
    map_item(s, blockIdx.x / (uint32_t)parts.splits, items / (uint32_t)parts.splits, row_tiles, true,
             slice, tile_at);
    const int row0 = tile_at * (16 * NR), row_n = min(16 * NR, s.rows - row0);
    const int b = (int)(slice / (uint32_t)s.kv_heads), a = (int)(slice - (uint32_t)b * s.kv_heads);
    int ql, kl;
    lengths(s, b, ql, kl);
    const int p0 = kl - ql;

    const int t_first = row0 / s.group, t_last = min((row0 + row_n - 1) / s.group, ql - 1);
    KeyList keys = {};
    if (t_first <= t_last) keys = key_list(s, p0 + t_first, p0 + t_last, kl);
    int slot_a = 0, slot_e = keys.count;
    if (parts.splits > 1) {
        const int per = ((keys.count + KT - 1) / KT + parts.splits - 1) / parts.splits * KT;
        slot_a = min(split * per, keys.count);
        slot_e = min(keys.count, slot_a + per);
    }
    const T* kb = k + (int64_t)b * s.k.batch + (int64_t)a * s.k.head;
    const T* vb = v + (int64_t)b * s.v.batch + (int64_t)a * s.v.head;

    Frag qf[NR][KS];
    Sight see[NR];
#pragma unroll
    for (int nr = 0; nr < NR; ++nr) {
        const int row = row0 + 16 * nr + l16, tok = row / s.group;
        const bool valid = row < s.rows && tok < ql;
        see[nr] = sight(s, keys, p0 + tok, kl, valid);
        const T* p = q + (int64_t)b * s.q.batch +
                     (int64_t)(a * s.group + (row - tok * s.group)) * s.q.head + (int64_t)tok * s.q.token;
#pragma unroll
        for (int ks = 0; ks < KS; ++ks)
            qf[nr][ks] = valid ? Mma<T>::load(p + 32 * ks + 8 * grp) : Frag{};
    }
    const RowsSight rows = rows_sight(s, keys, row0, row_n, p0, ql, kl);

    const float c2 = s.scale * kLog2e;
    f32x4 acc[NR][DT];
    float m_ref[NR], l_run[NR];
#pragma unroll
    for (int nr = 0; nr < NR; ++nr) {
        m_ref[nr] = kNoRef;
        l_run[nr] = 0.0f;
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) acc[nr][dt] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    }

    auto place = [](int row, int chunk) {
        return row * ROW + ((chunk ^ ((((row & 3) << 1) | ((row >> 2) & 1)) & (CHUNKS - 1))) << 4);
    };
    // Loads of 32 keys; slots past the end repeat the last key (its weight is 0).
    Frag kf[2][KS];
    i32x4 vr[V_LOADS];
    auto fetch = [&](int slot0) {
#pragma unroll
        for (int kt = 0; kt < 2; ++kt) {
            const T* p = kb + (int64_t)keys.row(min(slot0 + 16 * kt + l16, slot_e - 1)) * s.k.token;
#pragma unroll
            for (int ks = 0; ks < KS; ++ks) kf[kt][ks] = Mma<T>::load(p + 32 * ks + 8 * grp);
        }
#pragma unroll
        for (int i = 0; i < V_LOADS; ++i) {
            const int at = lane + 64 * i;
            const T* p = vb + (int64_t)keys.row(min(slot0 + at / CHUNKS, slot_e - 1)) * s.v.token;
            vr[i] = *(const i32x4*)((const char*)p + 16 * (at % CHUNKS));
        }
    };
    int slot0 = slot_a + KT * wave;
    if (slot0 < slot_e) fetch(slot0);
    for (; slot0 < slot_e; slot0 += KT * W) {
        lane_exchange();                               // (reads of the tile before)
#pragma unroll
        for (int i = 0; i < V_LOADS; ++i) {
            const int at = lane + 64 * i;
            *(i32x4*)(mine + place(at / CHUNKS, at % CHUNKS)) = vr[i];
        }
        f32x4 st[NR][2];
#pragma unroll
        for (int nr = 0; nr < NR; ++nr)
#pragma unroll
            for (int kt = 0; kt < 2; ++kt) {
                st[nr][kt] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
                for (int ks = 0; ks < KS; ++ks) st[nr][kt] = M::mul(kf[kt][ks], qf[nr][ks], st[nr][kt]);
            }
        lane_exchange();
        if (slot0 + KT * W < slot_e) fetch(slot0 + KT * W);

        const bool full = slot0 + KT <= slot_e && rows.all(slot0, KT);
        Frag p[NR];
#pragma unroll
        for (int nr = 0; nr < NR; ++nr) {
            if (!full) {
#pragma unroll
                for (int kt = 0; kt < 2; ++kt)
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        const int slot = slot0 + 16 * kt + 4 * grp + r;
                        const bool seen = slot < slot_e && see[nr].sees(slot);
                        st[nr][kt][r] = seen ? st[nr][kt][r] : -INFINITY;
                    }
            }
            f32x4 w[2];
            auto weights = [&]() -> float {
                float rs = 0.0f;
#pragma unroll
                for (int kt = 0; kt < 2; ++kt)
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        w[kt][r] = __builtin_amdgcn_exp2f(fmaf(st[nr][kt][r], c2, -m_ref[nr]));
                        rs += w[kt][r];
                    }
                return rs;
            };
            float rs = weights();
            if (__builtin_amdgcn_ballot_w64(!(rs <= kSumLimit)) != 0) {
                float mx = st[nr][0][0];
#pragma unroll
                for (int i = 1; i < 8; ++i) mx = fmaxf(mx, st[nr][i >> 2][i & 3]);
                const float m_new = fmaxf(m_ref[nr], row_max16(mx) * c2);
                const float alpha = __builtin_amdgcn_exp2f(m_ref[nr] - m_new);
                m_ref[nr] = m_new;
                l_run[nr] *= alpha;
#pragma unroll
                for (int dt = 0; dt < DT; ++dt) acc[nr][dt] *= alpha;
                rs = weights();
            }
            l_run[nr] += rs;
            p[nr] = M::pack(w[0], w[1]);
        }
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) {
            // V transposed: channel 16 dt + l16, keys 4 grp .. + 3 of both halves
            Frag f;
            if constexpr (sizeof(T) == 2) {
                bf16x4 part[2];
#pragma unroll
                for (int kt = 0; kt < 2; ++kt) {
                    const int row = 16 * kt + 4 * grp + (l16 >> 2), col = 16 * dt + 4 * (l16 & 3);
                    part[kt] = __builtin_amdgcn_ds_read_tr16_b64_v4bf16(
                        LDS_PTR(bf16x4, mine + place(row, col >> 3) + (col & 7) * 2));
                }
                f = __builtin_shufflevector(part[0], part[1], 0, 1, 2, 3, 4, 5, 6, 7);
            } else {
                const int d = 16 * dt + l16;
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    f[i] = *(const float*)(mine + place(16 * (i >> 2) + 4 * grp + (i & 3), d >> 2) +
                                           (d & 3) * 4);
            }
#pragma unroll
            for (int nr = 0; nr < NR; ++nr) acc[nr][dt] = M::mul(f, p[nr], acc[nr][dt]);
        }
    }

    // ---- the wavefronts' sums, each against the largest reference, in their order
#pragma unroll
    for (int nr = 0; nr < NR; ++nr) {
        const float l = row_sum16(l_run[nr]);
        if (grp == 0) {
            m_s[wave][16 * nr + l16] = m_ref[nr];
            l_s[wave][16 * nr + l16] = l;
        }
    }
    __syncthreads();                                   // (the V tiles are used up as well)
#pragma unroll
    for (int nr = 0; nr < NR; ++nr) {
        float top = kNoRef;
#pragma unroll
        for (int w = 0; w < W; ++w) top = fmaxf(top, m_s[w][16 * nr + l16]);
        const float f = __builtin_amdgcn_exp2f(m_ref[nr] - top);
#pragma unroll
        for (int dt = 0; dt < DT; ++dt)
            *(f32x4*)(mine + ((16 * nr + l16) * D + 16 * dt + 4 * grp) * 4) = acc[nr][dt] * f;
    }
    __syncthreads();
    const int quads = row_n * (D / 4);
    for (int at = tid; at < quads; at += 64 * W) {
        const int own = at / (D / 4), row = row0 + own, c = at % (D / 4) * 4;
        float top = kNoRef, l = 0.0f;
#pragma unroll
        for (int w = 0; w < W; ++w) top = fmaxf(top, m_s[w][own]);
        f32x4 sum = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int w = 0; w < W; ++w) {
            l = fmaf(__builtin_amdgcn_exp2f(m_s[w][own] - top), l_s[w][own], l);
            sum += *(const f32x4*)(lds + w * REGION + (own * D + c) * 4);
        }
        const int tok = row / s.group, head = a * s.group + (row - tok * s.group);
        if (parts.splits > 1) {
            const int64_t part = part_of(s, parts, slice, row, split);
            *(f32x4*)(parts.acc + part * D + c) = sum;
            if (c == 0) parts.ml[part] = make_float2(top, l);
        } else {
            const float f = l == 0.0f ? 0.0f : 1.0f / l;
            put4(out + (int64_t)b * s.out.batch + (int64_t)head * s.out.head +
                     (int64_t)tok * s.out.token + c,
                 sum[0] * f, sum[1] * f, sum[2] * f, sum[3] * f);
            if (lse && c == 0)
                lse[((int64_t)b * s.heads + head) * s.q_tokens + tok] =
                    l == 0.0f ? -INFINITY : (top + __builtin_amdgcn_logf(l)) * kLn2;
        }
    }
}

template <typename T, int D>
hipError_t launch_step(const Shape& s, const void* q, const void* k, const void* v, void* out,
                       float* lse, const Parts& parts, hipStream_t stream)
{
    const uint32_t row_tiles = s.rows <= 16 ? 1u : ((uint32_t)s.rows + 31) / 32;
    const uint32_t items = row_tiles * (uint32_t)(s.batch * s.kv_heads * parts.splits);
    constexpr int WIDE = step_waves(sizeof(T), D);
    const bool wide = is_wide_step(sizeof(T) == 2, D, s);
    auto kernel = s.rows > 16 ? window_step_kernel<T, D, 2, 4>
                  : wide      ? window_step_kernel<T, D, 1, WIDE>
                              : window_step_kernel<T, D, 1, 4>;
    kernel<<<items, 64 * (wide ? WIDE : 4), 0, stream>>>((const T*)q, (const T*)k, (const T*)v, (T*)out,
                                                         lse, s, parts, row_tiles, items);
    return hipGetLastError();
}

}  // namespace win

hipError_t launch_window_step(bool is_bf16, int D, const win::Shape& s, const void* q, const void* k,
                              const void* v, void* out, float* lse, const win::Parts& parts,
                              hipStream_t stream)
{
    using namespace win;
#define BSA_WINDOW_STEP(T, D_) launch_step<T, D_>(s, q, k, v, out, lse, parts, stream)
    if (is_bf16)
        return D == 32   ? BSA_WINDOW_STEP(uint16_t, 32)
               : D == 64 ? BSA_WINDOW_STEP(uint16_t, 64)
                         : BSA_WINDOW_STEP(uint16_t, 128);
    return D == 32   ? BSA_WINDOW_STEP(float, 32)
           : D == 64 ? BSA_WINDOW_STEP(float, 64)
                     : BSA_WINDOW_STEP(float, 128);
#undef BSA_WINDOW_STEP
}

}  // namespace bsa
