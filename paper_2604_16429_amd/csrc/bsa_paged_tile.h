// Attention over a cache in pages for many rows, bf16, head dims 64 and 128: four wavefronts own 128 rows
// and walk a list of tokens in tiles of 64 that all of them read from LDS (bsa_window_walk.h).
//
// Tiles are gathered straight into LDS, 1 KiB (4 or 8 rows) by a load, whose rows lie in one page: its address
// is scalar.  A lane holds the page of one token of the tile, asked for a tile before it is needed.  Rows that
// are not there repeat the last one, those of entries that name no page are zeros; both are hidden in
// what S^T starts from.  Scalar registers are short: pages of 64 tokens and more have a kernel of their own, which
// needs one address a tile (two sequences of 8,192 read in, pages of 128: 1,105 us; with an address for each
// load 1,265, with all forms in one kernel 1,160).
#pragma once

#include "bsa_paged.h"
#include "bsa_window_walk.h"

namespace bsa {

namespace paged {

// Whether 31 bits reach from the first to the last row of a tile and 32 hold a page's stride.
inline bool strides_fit(const Shape& s)
{
    return s.k.token < 1 << 24 && s.v.token < 1 << 24 && s.k.batch >> 32 == 0 && s.v.batch >> 32 == 0;
}

// ONE: pages of 64 tokens and more, so that a tile lies in one.
template <int D, bool ONE>
struct WideTile {
    static constexpr int KT = 64, KS = D / 16, DT = D / 32;
    using R = win::Rows<D>;
    static constexpr int LDS_BYTES = (int)sizeof(typename win::Walk<D>::Tiles);
    static constexpr int MINE = KT / R::PER_SLAB / 4;  // loads of a wavefront for a tile

    // Tiles t_a .. t_e - 1 for the given rows; part as in Step.
    static __device__ __forceinline__ void walk(unsigned char* lds, const Args<uint16_t>& g, const Rows& rows,
                                                const Sequence& seq, const Tiles<KT>& list, int t_a, int t_e,
                                                int64_t part)
    {
        const Shape& s = g.s;
        auto& tiles_s = *(typename win::Walk<D>::Tiles*)lds;
        const int lane = threadIdx.x & 63;
        const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
        const int l32 = lane & 31, half = lane >> 5;
        const uint16_t* kb = g.k + (int64_t)rows.a * s.k.head;
        const uint16_t* vb = g.v + (int64_t)rows.a * s.v.head;
        const int32_t* own_table = s.table + (int64_t)max(rows.b, 0) * s.table_pages;
        const int in_page = (1 << s.page_shift) - 1;

        // A tile and, in every lane, the page of token `lane` of it: -1 if it names none, the last token's behind
        // the list's end.  n: its tokens, at most KT of them count; 0: no tile.
        struct Ahead {
            int at, n, token, id;
        };
        auto ask = [&](int t) -> Ahead {
            Ahead x = {0, 0, 0, -1};
            if (t < t_e) {
                const Tile tile = list[t];
                const int32_t* table = tile.shared ? s.prefix_table : own_table;
                x.at = tile.at;
                x.n = tile.count - tile.at;
                x.token = tile.token;
                x.id = page_of(s, table, min(tile.at + lane, tile.count - 1), tile.count);
            }
            return x;
        };
        auto hidden_of = [&](const Ahead& x) -> uint64_t { return __builtin_amdgcn_ballot_w64(x.id < 0 || lane >= x.n); };
        const int row_of = lane / R::CHUNKS;           // of this lane in a load
        const uint32_t chunk = (uint32_t)R::swizzled(row_of, lane % R::CHUNKS) * 16;
        // (strides_fit: 32-bit strides)
        auto row_at_page = [&](const uint16_t* pool, const mosaic_bsa_strides& st, int page, int at) {
            return pool + (uint64_t)(uint32_t)page * (uint32_t)st.batch +
                   (uint64_t)(uint32_t)(at & in_page) * (uint32_t)st.token;
        };
        auto gather = [&](const uint16_t* pool, const mosaic_bsa_strides& st, const Ahead& x, uint64_t hidden,
                          unsigned char* to) {
            const int n = x.n, id = x.id;
            if (n <= 0) return;
            const uint32_t stride = (uint32_t)st.token * 2u, to0 = lds_address(to) + (uint32_t)(wave * R::SLAB);
            auto nothing = [&](int i) { *(uint4*)(to + (wave + 4 * i) * R::SLAB + 16 * lane) = make_uint4(0, 0, 0, 0); };
            if constexpr (ONE) {
                const int page = __builtin_amdgcn_readfirstlane(id);
                if (page < 0) {
#pragma unroll
                    for (int i = 0; i < MINE; ++i) nothing(i);
                    return;
                }
                const i32x4 rsrc = buffer_desc(row_at_page(pool, st, page, x.at), (KT - 1) * stride + R::ROW_BYTES);
                const int row = R::PER_SLAB * wave + row_of;
                if (n >= KT) {
                    const uint32_t from = (uint32_t)row * stride + chunk;
#pragma unroll
                    for (int i = 0; i < MINE; ++i)
                        load_lds_16(rsrc, from, (uint32_t)(4 * R::PER_SLAB * i) * stride, to0 + (uint32_t)(4 * i * R::SLAB));
                } else {
#pragma unroll
                    for (int i = 0; i < MINE; ++i)
                        load_lds_16(rsrc, (uint32_t)min(row + 4 * R::PER_SLAB * i, n - 1) * stride + chunk, 0,
                                    to0 + (uint32_t)(4 * i * R::SLAB));
                }
            } else if (hidden == 0) {
                const uint32_t from = (uint32_t)row_of * stride + chunk;
#pragma unroll
                for (int i = 0; i < MINE; ++i) {
                    const int r0 = R::PER_SLAB * (wave + 4 * i);
                    const uint16_t* p = row_at_page(pool, st, __builtin_amdgcn_readlane(id, r0), x.at + r0);
                    load_lds_16(buffer_desc(p, (R::PER_SLAB - 1) * stride + R::ROW_BYTES), from, 0,
                                to0 + (uint32_t)(4 * i * R::SLAB));
                }
            } else {
#pragma unroll
                for (int i = 0; i < MINE; ++i) {
                    const int r0 = min(R::PER_SLAB * (wave + 4 * i), n - 1);
                    const int page = __builtin_amdgcn_readlane(id, r0);
                    if (page < 0) {
                        nothing(i);
                        continue;
                    }
                    const uint32_t r = (uint32_t)min(row_of, n - 1 - r0);
                    load_lds_16(buffer_desc(row_at_page(pool, st, page, x.at + r0), (R::PER_SLAB - 1) * stride + R::ROW_BYTES),
                                r * stride + chunk, 0, to0 + (uint32_t)(4 * i * R::SLAB));
                }
            }
        };
        auto k_to = [&](int t) { return tiles_s[0][(t - t_a) & 1]; };
        auto v_to = [&](int t) { return tiles_s[1][(t - t_a) & 1]; };
        // the next two tiles, with their hidden tokens, and what masks of the present one take
        Ahead next = ask(t_a), after = ask(t_a + 1);
        uint64_t hidden = hidden_of(next), next_hidden = hidden_of(after);
        int token = next.token;
        gather(kb, s.k, next, hidden, k_to(t_a));
        gather(vb, s.v, next, hidden, v_to(t_a));
        gather(kb, s.k, after, next_hidden, k_to(t_a + 1));
        next = after;
        after = ask(t_a + 2);

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
        bf16x8 qf[KS];
        {
            const uint16_t* p = g.q + (int64_t)x.b * s.q.batch + (int64_t)x.head * s.q.head +
                                (int64_t)x.tok * s.q.token + 8 * half;
#pragma unroll
            for (int ks = 0; ks < KS; ++ks) qf[ks] = query ? *(const bf16x8*)(p + 16 * ks) : bf16x8{};
        }
        f32x16 acc[DT];
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) acc[dt] = win::splat(0.0f);
        float m_ref = kNoRef, l_run = 0.0f;

        // (rows that are no query may see what they like: nothing is kept of them; behind the last tile there is
        // nothing to keep either)
        const int lo_all = last - s.left;
        auto full = [&](int, int h) -> bool {
            const int j = token + 32 * h;
            return (uint32_t)(hidden >> (32 * h)) == 0 && j + 31 <= first && (j >= lo_all || j + 32 <= s.sinks);
        };
        auto start = [&](int, int h) -> f32x16 {
            const int j = token + 32 * h + 4 * half;
            const uint32_t mask = (uint32_t)(hidden >> (32 * h)) >> (4 * half);
            const uint32_t lo = (uint32_t)(j - (place - s.left));
            const int sinks = min(s.sinks, place + 1) - j;
            f32x16 st;
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                const int c = 8 * (e >> 2) + (e & 3);
                const bool seen = (lo + (uint32_t)c <= (uint32_t)s.left || c < sinks) && !(mask >> c & 1u);
                st[e] = seen ? 0.0f : -INFINITY;
            }
            return st;
        };
        // (in the middle of a tile: its masks are done, those of the next one follow)
        win::walk_tiles<D>(tiles_s, t_a, t_e, qf, s.scale * kLog2e, acc, m_ref, l_run, lane, full, start, [&](int t) {
            token = next.token;
            hidden = next_hidden;
            next_hidden = hidden_of(after);
            gather(kb, s.k, after, next_hidden, k_to(t + 2));
            gather(vb, s.v, next, hidden, v_to(t + 1));
            next = after;
            after = ask(t + 3);
        });

        const float l = l_run + swap32(l_run);
        wait_gathers_and_reads();
        __syncthreads();                               // the tiles are used up
        if (part >= 0) {
            // through LDS, so that a store instruction writes 1 KiB on end (128 members on 131,072 shared
            // tokens, 33 MB of sums: 182 us straight from the accumulators, 176 so)
            unsigned char* const mine = lds + wave * 32 * D * 4;
#pragma unroll
            for (int dt = 0; dt < DT; ++dt)
#pragma unroll
                for (int r = 0; r < 4; ++r)
                    *(f32x4*)(mine + l32 * D * 4 + ((8 * dt + 2 * r + half) ^ (l32 & 15)) * 16) =
                        f32x4{acc[dt][4 * r], acc[dt][4 * r + 1], acc[dt][4 * r + 2], acc[dt][4 * r + 3]};
            lane_exchange();
            float* const to = g.plan.acc + (part + 32 * wave) * D;
            const int there = min(32, rows.n - 32 * wave) * (D / 4);
#pragma unroll
            for (int i = 0; i < D / 8; ++i) {
                const int at = 64 * i + lane, r = at / (D / 4), c = at % (D / 4);
                if (at < there) *(f32x4*)(to + 4 * at) = *(const f32x4*)(mine + r * D * 4 + (c ^ (r & 15)) * 16);
            }
            if (exists && half == 0) g.plan.ml[part + 32 * wave + l32] = make_float2(m_ref, l);
            return;
        }
        const bool none = !query || l == 0.0f;
        if (none)
#pragma unroll
            for (int dt = 0; dt < DT; ++dt) acc[dt] = win::splat(0.0f);
        win::store_wave_rows<D>(g.out + (int64_t)rows.b * s.out.batch + (int64_t)rows.a * s.group * s.out.head, s.out,
                                s, rows.row0 + 32 * wave, acc, none ? 0.0f : 1.0f / l, lds + 4096 * wave, lane);
        if (g.lse && half == 0 && exists)
            g.lse[((int64_t)x.b * s.heads + x.head) * s.q_tokens + x.tok] =
                none ? -INFINITY : (m_ref + __builtin_amdgcn_logf(l)) * kLn2;
    }
};

}  // namespace paged

}  // namespace bsa
