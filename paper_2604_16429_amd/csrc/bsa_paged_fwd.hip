// Attention over a cache in pages: launches.  Which rows and tokens a workgroup takes is in
// bsa_paged_plan.h.
#include "bsa_paged_general.h"
#include "bsa_paged_step.h"
#include "bsa_paged_tile.h"

namespace bsa {

namespace paged {

constexpr int most_of(int a, int b) { return a > b ? a : b; }

// What works on tiles of ROWS rows.
template <typename T, int D, int ROWS, int W, bool ONE>
struct WalkOf {
    using Type = Step<T, D, ROWS / 16, W>;
};
template <typename T, int D, int W, bool ONE>
struct WalkOf<T, D, 128, W, ONE> {
    using Type = GeneralTile<T, D>;
};
template <int W, bool ONE>
struct WalkOf<uint16_t, 64, 128, W, ONE> {
    using Type = WideTile<64, ONE>;
};
template <int W, bool ONE>
struct WalkOf<uint16_t, 128, 128, W, ONE> {
    using Type = WideTile<128, ONE>;
};
// bf16 at head dims 64 and 128: tiles of 128 rows where the rows of a load share a page.  Else only from as many
// of them on, and of their tokens, as pay for giving up 32 rows whose tokens wavefronts share out.  us, 32 | 128 rows: bf16,
// head dim 32, 2 x 8,192 read in, 512 workgroups, 338 | 231, 2 x 2,048, 256, 19 | 28; fp32, head dim 64, 2 x
// 4,096, 1,024, 673 | 599, 16 x 40 on a prefix of 1,007, 256, 60 | 85, 4 x 1,796 on up to 7,090 tokens, 116, 252 | 217,
// 2 x 300 on up to 20,000, 20, 210 | 257; head dim 128, where 32 rows leave one wavefront a SIMD, 2 x 376 on 36,894 tokens,
// 48, 1,934 | 1,087, 64 on 3,000, 4, 26 | 48.
Kind kind_of(bool is_bf16, int D, const Shape& s, bool fit)
{
    // Tokens of up to 16 rows that stay in one workgroup.  us, in one | split: bf16, head dim 64, 16 slices, 1,000 tokens
    // 10.9 | 11.0, 2,000 15.5 | 11.1, 128 slices, 2,000 17 | 22, 4,000 26 | 30; head dim 128, 16 slices, 600 11.1 | 11.8,
    // 1,000 15.7 | 12.3; fp32, head dim 32, 16 slices, 600 9.8 | 11.1, 1,000 12.5 | 11.1, 128 slices, head dim 64, 600
    // 15 | 18.
    const int waves = win::step_waves(is_bf16 ? 2 : 4, D);
    const bool many = (int64_t)s.batch * s.kv_heads >= 128;
    Kind kind = {32, 32, waves, waves * (is_bf16 ? many ? 256 : 72 : many ? 128 : 48), 2 * D * (is_bf16 ? 2 : 4)};
    if (is_bf16 && D >= 64) {
        if (fit && (1 << s.page_shift) >= 1024 / (2 * D)) kind.most_own = kind.most_shared = 128;
    } else if (const int64_t tiles = (int64_t)s.batch * s.kv_heads * ((s.rows + 127) / 128);
               tiles >= (D == 128 ? 32 : most_tokens(s, false) >= 4096 ? 96 : 512)) {
        kind.most_own = 128;
    }
    return kind;
}
// Workgroups that a CU is to hold: as many as the registers of each kernel allow.
template <typename T, int D, int ROWS, int W>
constexpr int held_by_cu()
{
    return W > 4 || sizeof(T) == 4 ? 1 : ROWS == 128 && D == 64 ? 3 : 2;
}

// OWN, SHARED: rows of a workgroup that takes a sequence's, and of one that takes those of all (0: none does).
template <typename T, int D, int OWN, int SHARED, int W, bool ONE = false>
__global__ __launch_bounds__(64 * W, (held_by_cu<T, D, most_of(OWN, SHARED), W>())) void paged_kernel(
    const Args<T> g, uint32_t shared_items)
{
    using Own = typename WalkOf<T, D, OWN, W, ONE>::Type;
    using Shared = typename WalkOf<T, D, SHARED ? SHARED : 16, W, ONE>::Type;
    __shared__ __attribute__((aligned(1024))) unsigned char
        lds[SHARED ? most_of(Own::LDS_BYTES, Shared::LDS_BYTES) : Own::LDS_BYTES];
    const Shape& s = g.s;
    const Plan& plan = g.plan;
    const int lane = threadIdx.x & 63;

    if (SHARED && blockIdx.x < shared_items) {
        const uint32_t item = blockIdx.x, rest = item / (uint32_t)plan.shared_splits;
        const int split = (int)(item - rest * (uint32_t)plan.shared_splits);
        const int tile = (int)(rest / (uint32_t)s.kv_heads);
        Rows rows;
        rows.a = (int)(rest - (uint32_t)tile * s.kv_heads);
        rows.b = -1;
        rows.row0 = tile * SHARED;
        rows.n = min(SHARED, plan.all_rows - rows.row0);
        Sequence seq = {0, 0, 0};
        seq.prefix = __builtin_amdgcn_readfirstlane(prefix_of(s));
        const Tiles<Shared::KT> tiles(s, seq, 0, seq.prefix - 1, kShared);
        const int per = (tiles.count + plan.shared_splits - 1) / plan.shared_splits;
        const int t_a = min(split * per, tiles.count);
        Shared::walk(lds, g, rows, seq, tiles, t_a, min(t_a + per, tiles.count),
                     plan.shared_part(s, rows.a, split, rows.row0));
        return;
    }
    const uint32_t item = blockIdx.x - (SHARED ? shared_items : 0u);
    const int w = (int)(item / (uint32_t)s.kv_heads);
    Rows rows;
    rows.a = (int)(item - (uint32_t)w * s.kv_heads);
    Chunk chunk = chunk_at(s, plan, w, lane,
                           plan.parts && rows.a == 0 && (w == 0 || !plan.scanned) && threadIdx.x < 64);
    chunk.entry = __builtin_amdgcn_readfirstlane(chunk.entry);
    chunk.first = __builtin_amdgcn_readfirstlane(chunk.first);
    chunk.chunks = __builtin_amdgcn_readfirstlane(chunk.chunks);
    if (chunk.entry < 0) return;
    rows.b = plan.sequence_of(s, chunk.entry);
    const int tile = plan.tile_of(s, chunk.entry);
    rows.row0 = tile * OWN;
    rows.n = min(OWN, s.rows - rows.row0);
    const Sequence seq = uniform(sequence(s, rows.b));
    const auto tiles = tiles_of<Own::KT>(s, plan, seq, tile);
    const int per = (tiles.count + chunk.chunks - 1) / chunk.chunks;
    const int t_a = min((w - chunk.first) * per, tiles.count);
    const bool direct = !SHARED && chunk.chunks == 1;
    Own::walk(lds, g, rows, seq, tiles, t_a, min(t_a + per, tiles.count), direct ? -1 : plan.own_part(rows.a, w));
}

// The parts of a row, each group's in their order, the prefix's first: out = sum 2^(m - M) acc / sum 2^(m - M) l.  A
// workgroup has rows of one sequence; D / 4 lanes have a row, PG groups of them take its parts in turn.
template <typename T, int D, int PG>
__global__ __launch_bounds__(256) void paged_join_kernel(const Args<T> g, uint32_t row_groups)
{
    constexpr int LANES = D / 4, PER = 256 / (LANES * PG);     // rows of a workgroup
    __shared__ f32x4 sum_s[PG][PER * LANES];
    __shared__ float2 ml_s[PG][PER * LANES];
    const Shape& s = g.s;
    const Plan& plan = g.plan;
    const int b = (int)(blockIdx.x / row_groups), tid = threadIdx.x;
    const int at = tid % LANES, slot = tid / LANES % PER, pg = tid / (LANES * PER);
    const int slice_row = (int)(blockIdx.x - (uint32_t)b * row_groups) * PER + slot;     // (key/value head, row)
    const int a = min(slice_row / s.rows, s.kv_heads - 1), row = slice_row - a * s.rows;
    const int tile = min(row, s.rows - 1) / plan.tile;
    const Entry entry = plan.found[plan.entry_of(s, b, tile)];
    const Row x = row_at(s, Rows{row, 1, a, b}, sequence(s, b), 0);
    float top = kNoRef, l = 0.0f;
    f32x4 sum = {0.0f, 0.0f, 0.0f, 0.0f};
    const auto add = [&](float m, float l_part, const f32x4& v) {
        const float most = fmaxf(top, m);
        const float f0 = __builtin_amdgcn_exp2f(top - most), f = __builtin_amdgcn_exp2f(m - most);
        top = most;
        l = fmaf(f, l_part, l * f0);
#pragma unroll
        for (int e = 0; e < 4; ++e) sum[e] = fmaf(f, v[e], sum[e] * f0);
    };
    // n parts from `first` on, each `step` rows behind the one before; AHEAD of them are asked for at once
    const auto take = [&](int64_t first, int64_t step, int n) {
        constexpr int AHEAD = 8;
        for (int i0 = pg; i0 < n; i0 += PG * AHEAD) {
            float2 ml[AHEAD];
            f32x4 v[AHEAD];
#pragma unroll
            for (int u = 0; u < AHEAD; ++u)
                if (i0 + PG * u < n) {
                    const int64_t part = first + (i0 + PG * u) * step;
                    ml[u] = plan.ml[part];
                    v[u] = *(const f32x4*)(plan.acc + part * D + 4 * at);
                }
#pragma unroll
            for (int u = 0; u < AHEAD; ++u)
                if (i0 + PG * u < n) add(ml[u].x, ml[u].y, v[u]);
        }
    };
    const bool exists = row < s.rows;
    if (plan.stacked) take(plan.shared_part(s, a, 0, b * s.rows + row), plan.all_rows, exists ? plan.shared_splits : 0);
    // (one chunk and nothing else: stored by its workgroup)
    const bool there = exists && (plan.stacked || entry.chunks != 1);
    take(plan.own_part(a, entry.first) + row - tile * plan.tile, plan.tile_rows, there ? entry.chunks : 0);
    if constexpr (PG > 1) {
        sum_s[pg][slot * LANES + at] = sum;
        ml_s[pg][slot * LANES + at] = make_float2(top, l);
        __syncthreads();
        if (pg > 0) return;
#pragma unroll
        for (int i = 1; i < PG; ++i) {
            const float2 ml = ml_s[i][slot * LANES + at];
            add(ml.x, ml.y, sum_s[i][slot * LANES + at]);
        }
    }
    if (!there) return;
    store_row<T, D>(g, x, 4 * at, sum, top, l);
}

template <typename T, int D>
hipError_t launch(const Shape& s, const void* q, const void* k, const void* v, void* out, float* lse,
                  void* workspace, hipStream_t stream)
{
    const Kind kind = kind_of(sizeof(T) == 2, D, s, strides_fit(s));
    Args<T> g = {(const T*)q, (const T*)k, (const T*)v, (T*)out, lse, s, make_plan(s, D, kind)};
    Plan& plan = g.plan;
    if (plan.parts) {
        const int64_t n = plan.all_parts(s);
        plan.acc = (float*)workspace;
        plan.ml = (float2*)(plan.acc + n * D);
        plan.found = (Entry*)(plan.ml + n);
    }
    const int own = plan.tile, shared = plan.shared_tile;
    const uint32_t own_items = (uint32_t)plan.chunks * s.kv_heads;
    const uint32_t shared_items =
        shared ? (uint32_t)plan.shared_splits * s.kv_heads * ((plan.all_rows + shared - 1) / shared) : 0u;
    constexpr int WAVES = win::step_waves(sizeof(T), D);
    void (*kernel)(const Args<T>, uint32_t) = nullptr;
    if (plan.waves > 4) kernel = paged_kernel<T, D, 16, 0, WAVES>;
    else if (shared == 0) kernel = own == 16 ? paged_kernel<T, D, 16, 0, 4> : paged_kernel<T, D, 32, 0, 4>;
    else if (shared == 16) kernel = paged_kernel<T, D, 16, 16, 4>;
    else kernel = own == 16 ? paged_kernel<T, D, 16, 32, 4> : paged_kernel<T, D, 32, 32, 4>;
    if constexpr (sizeof(T) == 2 && D >= 64) {
        const bool one = s.page_shift >= 6;
#define BSA_PAGED_WIDE(OWN, SHARED) (one ? paged_kernel<T, D, OWN, SHARED, 4, true> : paged_kernel<T, D, OWN, SHARED, 4>)
        if (shared == 0 && own == 128) kernel = BSA_PAGED_WIDE(128, 0);
        if (shared == 128)
            kernel = own == 16   ? BSA_PAGED_WIDE(16, 128)
                     : own == 32 ? BSA_PAGED_WIDE(32, 128)
                                 : BSA_PAGED_WIDE(128, 128);
#undef BSA_PAGED_WIDE
    } else {
        if (shared == 0 && own == 128) kernel = paged_kernel<T, D, 128, 0, 4>;
        if (shared == 32 && own == 128) kernel = paged_kernel<T, D, 128, 32, 4>;
    }
    kernel<<<own_items + shared_items, 64 * plan.waves, 0, stream>>>(g, shared_items);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || !plan.parts) return e;
    // as many groups as leave each some eight parts of a row
    const int parts = plan.shared_splits + plan.chunks / plan.entries, groups = parts > 40 ? 8 : parts > 8 ? 4 : 1;
    const int per = 256 / (D / 4 * groups);
    const uint32_t row_groups = (uint32_t)((s.kv_heads * s.rows + per - 1) / per);
    auto join = groups == 8   ? paged_join_kernel<T, D, 8>
                : groups == 4 ? paged_join_kernel<T, D, 4>
                              : paged_join_kernel<T, D, 1>;
    join<<<row_groups * (uint32_t)s.batch, 256, 0, stream>>>(g, row_groups);
    return hipGetLastError();
}

}  // namespace paged

size_t paged_fwd_workspace(bool is_bf16, int D, const paged::Shape& s)
{
    using namespace paged;
    // (which kernels run depends on strides as well: enough for both)
    size_t most = 0;
    for (const bool fit : {false, true}) {
        const Plan p = make_plan(s, D, kind_of(is_bf16, D, s, fit));
        const size_t n = p.parts ? (size_t)p.all_parts(s) * (D + 2) * sizeof(float) + p.entries * sizeof(Entry) : 0;
        if (n > most) most = n;
    }
    return most;
}

hipError_t launch_paged_fwd(bool is_bf16, int D, const paged::Shape& s, const void* q, const void* k,
                            const void* v, void* out, float* lse, void* workspace,
                            hipStream_t stream)
{
#define BSA_PAGED_FWD(T, D_) paged::launch<T, D_>(s, q, k, v, out, lse, workspace, stream)
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
