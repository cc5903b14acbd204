// Attention over a cache in pages for many rows, fp32 and head dim 32: four wavefronts own 128 rows and
// walk a list of tokens in tiles that all of them read from LDS, filled through registers, so that the next
// tile's loads are in flight while this one is worked on.
//
// Per 32 tokens x 32 rows: S^T = K Q^T (a lane holds one row and 16 tokens), the weights against a
// running reference in fp32, O^T += V^T P^T with the accumulator's registers as operand.  Matrix instructions
// and, at head dim 32, exponentials bound it.
#pragma once

#include "bsa_paged.h"

namespace bsa {

namespace paged {

template <typename T, int D>
struct GeneralTile {
    static constexpr int KT = sizeof(T) == 2 ? 64 : 32, KS = D / 16, DT = D / 32;
    using Tl = win::Tile<T, D, KT>;
    using M = win::Mma<T>;
    using Frag = typename M::Frag;
    static constexpr int LDS_BYTES = 2 * Tl::BYTES;

    // Tiles t_a .. t_e - 1 for the given rows; part as in Step.
    static __device__ __forceinline__ void walk(unsigned char* lds, const Args<T>& g, const Rows& rows,
                                                const Sequence& seq, const Tiles<KT>& list, int t_a, int t_e,
                                                int64_t part)
    {
        const Shape& s = g.s;
        unsigned char *const k_lds = lds, *const v_lds = lds + Tl::BYTES;
        const int tid = threadIdx.x, lane = tid & 63;
        const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
        const int l32 = lane & 31, half = lane >> 5;
        const T* kb = g.k + (int64_t)rows.a * s.k.head;
        const T* vb = g.v + (int64_t)rows.a * s.v.head;
        const int32_t* own_table = s.table + (int64_t)max(rows.b, 0) * s.table_pages;
        const int in_page = (1 << s.page_shift) - 1;

        const Row x = row_at(s, rows, seq, min(32 * wave + l32, rows.n - 1));
        const bool exists = 32 * wave + l32 < rows.n, query = exists && x.query;
        const int place = query ? x.place : -1;
        int first = query ? x.place : 1 << 30, last = query ? x.place : -(1 << 30);
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            first = min(first, __shfl_xor(first, o));
            last = max(last, __shfl_xor(last, o));
        }
        first = __builtin_amdgcn_readfirstlane(first);
        last = __builtin_amdgcn_readfirstlane(last);
        Frag qf[KS];
        {
            const T* p = g.q + (int64_t)x.b * s.q.batch + (int64_t)x.head * s.q.head + (int64_t)x.tok * s.q.token;
#pragma unroll
            for (int ks = 0; ks < KS; ++ks) qf[ks] = query ? M::load(p + 16 * ks + 8 * half) : Frag{};
        }
        const float c2 = s.scale * kLog2e;
        f32x16 acc[DT];
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) acc[dt] = win::splat(0.0f);
        float m_ref = kNoRef, l_run = 0.0f;

        // The page of token `lane` (modulo KT) of a tile: -1 if it names none, the last token's behind the
        // list's end.
        auto ask = [&](int t) -> int {
            const Tile tile = list[t];
            const int32_t* table = tile.shared ? s.prefix_table : own_table;
            return page_of(s, table, min(tile.at + (lane & (KT - 1)), tile.count - 1), tile.count);
        };
        Tl kt, vt;
        uint64_t hidden_next = 0;
        auto fetch = [&](int t, int id) {
            const Tile tile = list[t];
            const int n = tile.count - tile.at;
            hidden_next = __builtin_amdgcn_ballot_w64(id < 0 || (lane & (KT - 1)) >= n);
#pragma unroll
            for (int i = 0; i < Tl::PER_THREAD; ++i) {
                const int at = tid + 256 * i, r = min(at / Tl::CHUNKS, n - 1), chunk = at % Tl::CHUNKS;
                const int page = __shfl(id, r);
                const int64_t row = (tile.at + r) & in_page;
                const char* pk = (const char*)(kb + (int64_t)page * s.k.batch + row * s.k.token);
                const char* pv = (const char*)(vb + (int64_t)page * s.v.batch + row * s.v.token);
                kt.held[i] = page >= 0 ? *(const i32x4*)(pk + 16 * chunk) : i32x4{0, 0, 0, 0};
                vt.held[i] = page >= 0 ? *(const i32x4*)(pv + 16 * chunk) : i32x4{0, 0, 0, 0};
            }
        };
        int id_next = -1;
        if (t_a < t_e) {
            fetch(t_a, ask(t_a));
            if (t_a + 1 < t_e) id_next = ask(t_a + 1);
        }
        for (int t = t_a; t < t_e; ++t) {
            const int token = list[t].token;
            const uint64_t hidden = hidden_next;
            __syncthreads();                           // everyone is done with the tile before
            kt.put(k_lds, tid);
            vt.put(v_lds, tid);
            __syncthreads();
            if (t + 1 < t_e) {
                fetch(t + 1, id_next);
                if (t + 2 < t_e) id_next = ask(t + 2);
            }
#pragma unroll
            for (int hh = 0; hh < KT / 32; ++hh) {
                const int j0 = token + 32 * hh;
                const uint32_t mask = (uint32_t)(hidden >> (32 * hh));
                if (mask == 0xffffffffu || j0 > last) continue;
                const bool full = mask == 0 && j0 + 31 <= first && (j0 >= last - s.left || j0 + 32 <= s.sinks);
                f32x16 st = win::splat(0.0f);
#pragma unroll
                for (int ks = 0; ks < KS; ++ks) st = M::mul(Tl::row_frag(k_lds, 32 * hh, ks, lane), qf[ks], st);
                if (!full) {
#pragma unroll
                    for (int r = 0; r < 16; ++r) {
                        const int y = 8 * (r >> 2) + 4 * half + (r & 3), j = j0 + y;
                        const bool seen = j <= place && (j >= place - s.left || j < s.sinks) && !(mask >> y & 1u);
                        st[r] = seen ? st[r] : -INFINITY;
                    }
                }
                f32x16 w;
                auto weights = [&]() -> float {
                    float rs = 0.0f;
#pragma unroll
                    for (int r = 0; r < 16; ++r) {
                        w[r] = __builtin_amdgcn_exp2f(fmaf(st[r], c2, -m_ref));
                        rs += w[r];
                    }
                    return rs;
                };
                float rs = weights();
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
                    rs = weights();
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
        if (part >= 0) {
            const int64_t at = part + 32 * wave + l32;
            win::store_lane_row<float, D>(g.plan.acc + at * D, acc, 1.0f, half);
            if (half == 0) g.plan.ml[at] = make_float2(m_ref, l);
            return;
        }
        const bool none = !query || l == 0.0f;
        if (none)
#pragma unroll
            for (int dt = 0; dt < DT; ++dt) acc[dt] = win::splat(0.0f);
        win::store_lane_row<T, D>(g.out + (int64_t)x.b * s.out.batch + (int64_t)x.head * s.out.head +
                                      (int64_t)x.tok * s.out.token,
                                  acc, none ? 0.0f : 1.0f / l, half);
        if (g.lse && half == 0)
            g.lse[((int64_t)x.b * s.heads + x.head) * s.q_tokens + x.tok] =
                none ? -INFINITY : (m_ref + __builtin_amdgcn_logf(l)) * kLn2;
    }
};

}  // namespace paged

}  // namespace bsa
