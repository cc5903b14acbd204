// Attention over a cache in pages, any shape: a workgroup owns 16 or 32 rows (token, head of the
// group) of a (sequence, key/value head) slice and walks the tokens that they see.
//
// Four wavefronts take tiles of 32 tokens in turn and share nothing until the end: no barrier stands
// between a wavefront and its next loads, which are in flight while it works on the tile before.  Rows
// fill 16-wide matrix instructions: S^T = K Q^T, whose K operand is loaded from memory as the lanes
// hold it, and O^T += V^T P^T, where V goes through LDS of the wavefront's own to be read transposed.  At
// the end the wavefronts' sums meet in LDS in their order.
#include "bsa_paged.h"

namespace bsa {

namespace paged {

using win::Mma;
using win::Mma16;

// NR: 16-row tiles.
template <typename T, int D, int NR>
__global__ __launch_bounds__(256) void paged_step_kernel(const T* __restrict__ q, const T* __restrict__ k,
                                                         const T* __restrict__ v, T* __restrict__ out,
                                                         float* __restrict__ lse, const Shape s,
                                                         uint32_t row_tiles)
{
    constexpr int W = 4, KS = D / 32, DT = D / 16, KT = 32;
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

    const uint32_t slice = blockIdx.x / row_tiles;
    const int row0 = (int)(blockIdx.x - slice * row_tiles) * (16 * NR), row_n = min(16 * NR, s.rows - row0);
    const int b = (int)(slice / (uint32_t)s.kv_heads), a = (int)(slice - (uint32_t)b * s.kv_heads);
    const Sequence seq = sequence(s, b);
    const int p0 = seq.prefix + seq.kl - seq.ql;
    const int p_first = p0 + row0 / s.group;
    const int p_last = p0 + min((row0 + row_n - 1) / s.group, seq.ql - 1);
    Tiles<KT> tiles(s, seq, p_first, p_last);
    if (p_last < p_first) tiles.count = 0;

    const T* kb = k + (int64_t)a * s.k.head;
    const T* vb = v + (int64_t)a * s.v.head;
    const int32_t* own_table = s.table + (int64_t)b * s.table_pages;
    const int in_page = (1 << s.page_shift) - 1;

    Frag qf[NR][KS];
    int place[NR];                                     // of this lane's rows; -1: no row
#pragma unroll
    for (int nr = 0; nr < NR; ++nr) {
        const int row = row0 + 16 * nr + l16, tok = row / s.group;
        const bool valid = row < s.rows && tok < seq.ql;
        place[nr] = valid ? p0 + tok : -1;
        const T* p = q + (int64_t)b * s.q.batch +
                     (int64_t)(a * s.group + (row - tok * s.group)) * s.q.head + (int64_t)tok * s.q.token;
#pragma unroll
        for (int ks = 0; ks < KS; ++ks)
            qf[nr][ks] = valid ? Mma<T>::load(p + 32 * ks + 8 * grp) : Frag{};
    }

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

    auto lds_at = [](int row, int chunk) {
        return row * ROW + ((chunk ^ ((((row & 3) << 1) | ((row >> 2) & 1)) & (CHUNKS - 1))) << 4);
    };
    // Loads of a tile; tokens that are not there, or whose page is none, are zeros and bits of `hidden`.
    Frag kf[2][KS];
    i32x4 vr[V_LOADS];
    uint32_t hidden_next = 0;
    auto fetch = [&](int t) {
        const Tile tile = tiles[t];
        const int32_t* table = tile.shared ? s.prefix_table : own_table;
        hidden_next = 0;
#pragma unroll
        for (int kt = 0; kt < 2; ++kt) {
            const int at = tile.at + 16 * kt + l16, id = page_of(s, table, at, tile.count);
            const T* p = kb + (int64_t)id * s.k.batch + (int64_t)(at & in_page) * s.k.token;
#pragma unroll
            for (int ks = 0; ks < KS; ++ks)
                kf[kt][ks] = id >= 0 ? Mma<T>::load(p + 32 * ks + 8 * grp) : Frag{};
            hidden_next |= (uint32_t)(__builtin_amdgcn_ballot_w64(id < 0) & 0xffffu) << (16 * kt);
        }
#pragma unroll
        for (int i = 0; i < V_LOADS; ++i) {
            const int x = lane + 64 * i, at = tile.at + x / CHUNKS;
            const int id = page_of(s, table, at, tile.count);
            const T* p = vb + (int64_t)id * s.v.batch + (int64_t)(at & in_page) * s.v.token;
            vr[i] = id >= 0 ? *(const i32x4*)((const char*)p + 16 * (x % CHUNKS)) : i32x4{0, 0, 0, 0};
        }
    };
    int t = wave;
    if (t < tiles.count) fetch(t);
    for (; t < tiles.count; t += W) {
        const int token = tiles[t].token;
        const uint32_t hidden = hidden_next;
        lane_exchange();                               // (reads of the tile before)
#pragma unroll
        for (int i = 0; i < V_LOADS; ++i) {
            const int x = lane + 64 * i;
            *(i32x4*)(mine + lds_at(x / CHUNKS, x % CHUNKS)) = vr[i];
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
        if (t + W < tiles.count) fetch(t + W);

        // all rows see all of it (rows that are none may see what they like: nothing is kept of them)
        const bool full = hidden == 0 && token + KT - 1 <= p_first &&
                          (token >= p_last - s.left || token + KT <= s.sinks);
        Frag p[NR];
#pragma unroll
        for (int nr = 0; nr < NR; ++nr) {
            if (!full) {
#pragma unroll
                for (int kt = 0; kt < 2; ++kt)
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        const int x = 16 * kt + 4 * grp + r, j = token + x;
                        const bool seen = j <= place[nr] && (j >= place[nr] - s.left || j < s.sinks) &&
                                          !(hidden >> x & 1u);
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
                const float m_new = fmaxf(m_ref[nr], win::row_max16(mx) * c2);
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
            // V transposed: channel 16 dt + l16, tokens 4 grp .. + 3 of both halves
            Frag f;
            if constexpr (sizeof(T) == 2) {
                bf16x4 part[2];
#pragma unroll
                for (int kt = 0; kt < 2; ++kt) {
                    const int row = 16 * kt + 4 * grp + (l16 >> 2), col = 16 * dt + 4 * (l16 & 3);
                    part[kt] = __builtin_amdgcn_ds_read_tr16_b64_v4bf16(
                        LDS_PTR(bf16x4, mine + lds_at(row, col >> 3) + (col & 7) * 2));
                }
                f = __builtin_shufflevector(part[0], part[1], 0, 1, 2, 3, 4, 5, 6, 7);
            } else {
                const int d = 16 * dt + l16;
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    f[i] = *(const float*)(mine + lds_at(16 * (i >> 2) + 4 * grp + (i & 3), d >> 2) +
                                           (d & 3) * 4);
            }
#pragma unroll
            for (int nr = 0; nr < NR; ++nr) acc[nr][dt] = M::mul(f, p[nr], acc[nr][dt]);
        }
    }

    // ---- the wavefronts' sums, each against the largest reference, in their order
#pragma unroll
    for (int nr = 0; nr < NR; ++nr) {
        const float l = win::row_sum16(l_run[nr]);
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
        const int tok = row / s.group, head = a * s.group + (row - tok * s.group);
        float top = kNoRef, l = 0.0f;
#pragma unroll
        for (int w = 0; w < W; ++w) top = fmaxf(top, m_s[w][own]);
        f32x4 sum = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int w = 0; w < W; ++w) {
            l = fmaf(__builtin_amdgcn_exp2f(m_s[w][own] - top), l_s[w][own], l);
            sum += *(const f32x4*)(lds + w * REGION + (own * D + c) * 4);
        }
        const bool none = tok >= seq.ql || l == 0.0f;
        const float f = 1.0f / l;
        put4(out + (int64_t)b * s.out.batch + (int64_t)head * s.out.head + (int64_t)tok * s.out.token + c,
             none ? 0.0f : sum[0] * f, none ? 0.0f : sum[1] * f, none ? 0.0f : sum[2] * f,
             none ? 0.0f : sum[3] * f);
        if (lse && c == 0)
            lse[((int64_t)b * s.heads + head) * s.q_tokens + tok] =
                none ? -INFINITY : (top + __builtin_amdgcn_logf(l)) * kLn2;
    }
}

template <typename T, int D>
hipError_t launch(const Shape& s, const void* q, const void* k, const void* v, void* out, float* lse,
                  hipStream_t stream)
{
    const uint32_t row_tiles = s.rows <= 16 ? 1u : ((uint32_t)s.rows + 31) / 32;
    const uint32_t items = row_tiles * (uint32_t)(s.batch * s.kv_heads);
    auto kernel = s.rows <= 16 ? paged_step_kernel<T, D, 1> : paged_step_kernel<T, D, 2>;
    kernel<<<items, 256, 0, stream>>>((const T*)q, (const T*)k, (const T*)v, (T*)out, lse, s, row_tiles);
    return hipGetLastError();
}

}  // namespace paged

size_t paged_fwd_workspace(bool is_bf16, int D, const paged::Shape& s) { return 0; }

hipError_t launch_paged_fwd(bool is_bf16, int D, const paged::Shape& s, const void* q, const void* k,
                            const void* v, void* out, float* lse, void* workspace,
                            hipStream_t stream)
{
#define BSA_PAGED_FWD(T, D_) paged::launch<T, D_>(s, q, k, v, out, lse, stream)
    if (is_bf16)
        return D == 32   ? BSA_PAGED_FWD(uint16_t, 32)
               : D == 64 ? BSA_PAGED_FWD(uint16_t, 64)
                         : BSA_PAGED_FWD(uint16_t, 128);
    return D == 32   ? BSA_PAGED_FWD(float, 32)
           : D == 64 ? BSA_PAGED_FWD(float, 64)
                     : BSA_PAGED_FWD(float, 128);
#undef BSA_PAGED_FWD
}

}  // namespace bsa
