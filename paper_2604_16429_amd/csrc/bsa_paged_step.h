// Attention over a cache in pages for few rows, any shape: W wavefronts own 16 or 32 rows and walk a list
// of tokens.
//
// The wavefronts take tiles of 32 tokens in turn and share nothing until the end: no barrier stands
// between a wavefront and its next loads, which are in flight while it works on the tile before.  Rows
// fill 16-wide matrix instructions: S^T = K Q^T, whose K operand is loaded from memory as the lanes
// hold it, and O^T += V^T P^T, where V goes through LDS of the wavefront's own to be read transposed.  At
// the end the wavefronts' sums meet in LDS in their order.
//
// A lane holds the page of one token of the tile after next.  Where pages have 16 tokens at least and the
// whole tile is there, a load's rows lie in one page, whose address is scalar; the last tile of a list,
// smaller pages and entries that name none are gathered row by row.
#pragma once

#include "bsa_paged.h"

namespace bsa {

namespace paged {

using win::Mma;
using win::Mma16;

template <typename T, int D, int NR, int W>
struct Step {
    static constexpr int KS = D / 32, DT = D / 16, KT = 32;
    static constexpr int ROW = D * sizeof(T), CHUNKS = ROW / 16;
    static constexpr int V_LOADS = KT * CHUNKS / 64, V_ROWS = 64 / CHUNKS;      // rows of a load
    static constexpr int ACC_BYTES = NR * 16 * D * 4;
    static constexpr int REGION = KT * ROW > ACC_BYTES ? KT * ROW : ACC_BYTES;    // of a wavefront
    static constexpr int SUMS = W * REGION, LDS_BYTES = SUMS + 2 * W * NR * 16 * 4;
    using Frag = typename Mma<T>::Frag;
    using M = Mma16<T>;

    static __device__ __forceinline__ int lds_at(int row, int chunk)
    {
        return row * ROW + ((chunk ^ ((((row & 3) << 1) | ((row >> 2) & 1)) & (CHUNKS - 1))) << 4);
    }

    // Four channels of a row's sums: 16 rows' same channels lie in different banks (without that, and with
    // rows that are none, the sums of 16 wavefronts took 3 us)
    static __device__ __forceinline__ int sums_at(int row, int quad)
    {
        return row * D * 4 + ((quad ^ (row & (D / 4 < 16 ? D / 4 - 1 : 15))) << 4);
    }

    // Tiles t_a .. t_e - 1 for the given rows.  part: index of the first row's sums; negative: these are
    // all of them, the rows are stored.
    static __device__ __forceinline__ void walk(unsigned char* lds, const Args<T>& g, const Rows& rows,
                                                const Sequence& seq, const Tiles<KT>& tiles, int t_a, int t_e,
                                                int64_t part)
    {
        const Shape& s = g.s;
        const int tid = threadIdx.x, lane = tid & 63;
        const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
        const int l16 = lane & 15, grp = lane >> 4;
        unsigned char* const mine = lds + wave * REGION;
        float* const m_s = (float*)(lds + SUMS);       // [NR * 16][W]
        float* const l_s = m_s + W * NR * 16;

        const T* kb = g.k + (int64_t)rows.a * s.k.head;
        const T* vb = g.v + (int64_t)rows.a * s.v.head;
        const int32_t* own_table = s.table + (int64_t)max(rows.b, 0) * s.table_pages;
        const int in_page = (1 << s.page_shift) - 1;

        Frag qf[NR][KS];
        int place[NR];                                 // of this lane's rows; -1: no query
        // the least and the largest place of a query
        int first = 1 << 30, last = -(1 << 30);
        if (rows.b >= 0) {
            const int p0 = seq.prefix + seq.kl - seq.ql;
            first = p0 + rows.row0 / s.group;
            last = p0 + min((rows.row0 + rows.n - 1) / s.group, seq.ql - 1);
        }
#pragma unroll
        for (int nr = 0; nr < NR; ++nr) {
            const int r = 16 * nr + l16;
            Row x = row_at(s, rows, seq, min(r, rows.n - 1));
            const bool valid = r < rows.n && x.query;
            place[nr] = valid ? x.place : -1;
            if (rows.b < 0) {
                first = valid ? min(first, x.place) : first;
                last = valid ? max(last, x.place) : last;
            }
            const T* p = g.q + (int64_t)x.b * s.q.batch + (int64_t)x.head * s.q.head + (int64_t)x.tok * s.q.token;
#pragma unroll
            for (int ks = 0; ks < KS; ++ks)
                qf[nr][ks] = valid ? Mma<T>::load(p + 32 * ks + 8 * grp) : Frag{};
        }

        if (rows.b < 0) {
#pragma unroll
            for (int o = 1; o < 16; o <<= 1) {
                first = min(first, __shfl_xor(first, o));
                last = max(last, __shfl_xor(last, o));
            }
            first = __builtin_amdgcn_readfirstlane(first);
            last = __builtin_amdgcn_readfirstlane(last);
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

        // The page of token `lane & 31` of a tile: -1 if it names none, the last token's behind the list's end.
        auto ask = [&](int t) -> int {
            const Tile tile = tiles[t];
            const int32_t* table = tile.shared ? s.prefix_table : own_table;
            return page_of(s, table, min(tile.at + (lane & 31), tile.count - 1), tile.count);
        };
        // Loads of a tile whose pages are in `id`.  Tokens that are not there are bits of `hidden`; what is
        // loaded for them is the last token, or zeros.
        Frag kf[2][KS];
        i32x4 vr[V_LOADS];
        uint32_t hidden_next = 0;
        const bool rows_in_page = s.page_shift >= 4 && s.k.token < 1 << 24 && s.v.token < 1 << 24;
        const uint32_t k_off = ((uint32_t)l16 * (uint32_t)s.k.token + 8u * grp) * (uint32_t)sizeof(T);
        const uint32_t v_off = (uint32_t)(lane / CHUNKS) * (uint32_t)s.v.token * (uint32_t)sizeof(T) + lane % CHUNKS * 16u;
        auto fetch = [&](int t, int id) {
            const Tile tile = tiles[t];
            const int n = tile.count - tile.at;
            hidden_next = (uint32_t)__builtin_amdgcn_ballot_w64(id < 0 || (lane & 31) >= n);
            if (rows_in_page && hidden_next == 0) {
                const T* base_k[2];
                const T* base_v[2];
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const int64_t page = __builtin_amdgcn_readlane(id, 16 * h);
                    const int row = (tile.at + 16 * h) & in_page;
                    base_k[h] = kb + page * s.k.batch + row * s.k.token;
                    base_v[h] = vb + page * s.v.batch + row * s.v.token;
                }
#pragma unroll
                for (int kt = 0; kt < 2; ++kt)
#pragma unroll
                    for (int ks = 0; ks < KS; ++ks)
                        kf[kt][ks] = Mma<T>::load((const T*)((const char*)(base_k[kt] + 32 * ks) + k_off));
#pragma unroll
                for (int i = 0; i < V_LOADS; ++i) {
                    const int r = V_ROWS * i;
                    vr[i] = *(const i32x4*)((const char*)(base_v[r >> 4] + (r & 15) * s.v.token) + v_off);
                }
            } else {
#pragma unroll
                for (int kt = 0; kt < 2; ++kt) {
                    const int r = min(16 * kt + l16, n - 1), page = __shfl(id, r);
                    const T* p = kb + (int64_t)page * s.k.batch + (int64_t)((tile.at + r) & in_page) * s.k.token;
#pragma unroll
                    for (int ks = 0; ks < KS; ++ks)
                        kf[kt][ks] = page >= 0 ? Mma<T>::load(p + 32 * ks + 8 * grp) : Frag{};
                }
#pragma unroll
                for (int i = 0; i < V_LOADS; ++i) {
                    const int r = min(V_ROWS * i + lane / CHUNKS, n - 1), page = __shfl(id, r);
                    const T* p = vb + (int64_t)page * s.v.batch + (int64_t)((tile.at + r) & in_page) * s.v.token;
                    vr[i] = page >= 0 ? *(const i32x4*)((const char*)p + lane % CHUNKS * 16) : i32x4{0, 0, 0, 0};
                }
            }
        };
        int t = t_a + wave, id_next = -1;
        if (t < t_e) {
            fetch(t, ask(t));
            if (t + W < t_e) id_next = ask(t + W);
        }
        for (; t < t_e; t += W) {
            const int token = tiles[t].token;
            const uint32_t hidden = hidden_next;
            lane_exchange();                           // (reads of the tile before)
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
            if (t + W < t_e) {
                fetch(t + W, id_next);
                if (t + 2 * W < t_e) id_next = ask(t + 2 * W);
            }

            // all rows see all of it (rows that are none may see what they like: nothing is kept of them)
            const bool full = hidden == 0 && token + KT - 1 <= first &&
                              (token >= last - s.left || token + KT <= s.sinks);
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
        auto of_row = [&](const float* at, int r, float (&x)[W]) {
#pragma unroll
            for (int w = 0; w < W; w += 4) {
                const f32x4 v = *(const f32x4*)(at + r * W + w);
#pragma unroll
                for (int e = 0; e < 4; ++e) x[w + e] = v[e];
            }
        };
        auto top_of = [&](int r) -> float {
            float m[W], top = kNoRef;
            of_row(m_s, r, m);
#pragma unroll
            for (int w = 0; w < W; ++w) top = fmaxf(top, m[w]);
            return top;
        };
#pragma unroll
        for (int nr = 0; nr < NR; ++nr)
            if (grp == 0) m_s[(16 * nr + l16) * W + wave] = m_ref[nr];
        __syncthreads();                               // (the V tiles are used up as well)
#pragma unroll
        for (int nr = 0; nr < NR; ++nr) {
            const float f = __builtin_amdgcn_exp2f(m_ref[nr] - top_of(16 * nr + l16));
            const float l = win::row_sum16(l_run[nr]) * f;
            if (grp == 0) l_s[(16 * nr + l16) * W + wave] = l;
            if (16 * nr + l16 < rows.n)
#pragma unroll
                for (int dt = 0; dt < DT; ++dt)
                    *(f32x4*)(mine + sums_at(16 * nr + l16, 4 * dt + grp)) = acc[nr][dt] * f;
        }
        __syncthreads();
        const int quads = rows.n * (D / 4);
        for (int at = tid; at < quads; at += 64 * W) {
            const int r = at / (D / 4), c = at % (D / 4) * 4;
            const float top = top_of(r);
            float ls[W], l = 0.0f;
            of_row(l_s, r, ls);
            f32x4 sum = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
            for (int w = 0; w < W; ++w) {
                l += ls[w];
                sum += *(const f32x4*)(lds + w * REGION + sums_at(r, c / 4));
            }
            if (part < 0) store_row<T, D>(g, row_at(s, rows, seq, r), c, sum, top, l);
            else store_part<D>(g.plan, part + r, c, sum, top, l);
        }
    }
};

}  // namespace paged

}  // namespace bsa
