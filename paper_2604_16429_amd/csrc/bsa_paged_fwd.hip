// Attention over a cache in pages: launches.  Which rows and tokens a workgroup takes is in
// bsa_paged_plan.h.
#include "bsa_paged_step.h"

namespace bsa {

namespace paged {

constexpr int most_of(int a, int b) { return a > b ? a : b; }

// OWN, SHARED: 16-row tiles of a workgroup that takes a sequence's rows, and the rows of all (0: none do).
template <typename T, int D, int OWN, int SHARED, int W>
__global__ __launch_bounds__(64 * W) void paged_kernel(const Args<T> g, uint32_t shared_items)
{
    using Own = Step<T, D, OWN, W>;
    using Shared = Step<T, D, most_of(SHARED, 1), W>;
    __shared__ __attribute__((aligned(1024))) unsigned char
        lds[SHARED ? most_of(Own::LDS_BYTES, Shared::LDS_BYTES) : Own::LDS_BYTES];
    const Shape& s = g.s;
    const Plan& plan = g.plan;
    const int lane = threadIdx.x & 63;

    if (SHARED && blockIdx.x < shared_items) {
        const uint32_t rest = blockIdx.x / (uint32_t)plan.shared_splits;
        const int split = (int)(blockIdx.x - rest * (uint32_t)plan.shared_splits);
        const int tile = (int)(rest / (uint32_t)s.kv_heads);
        Rows rows;
        rows.a = (int)(rest - (uint32_t)tile * s.kv_heads);
        rows.b = -1;
        rows.row0 = tile * 16 * SHARED;
        rows.n = min(16 * SHARED, plan.all_rows - rows.row0);
        Sequence seq = {0, 0, 0};
        seq.prefix = __builtin_amdgcn_readfirstlane(prefix_of(s));
        const Tiles<32> tiles(s, seq, 0, seq.prefix - 1, kShared);
        const Row x = row_at(s, rows, seq, min(lane, rows.n - 1));
        int first = x.query ? x.place : 1 << 30;
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) first = min(first, __shfl_xor(first, o));
        const int per = (tiles.count + plan.shared_splits - 1) / plan.shared_splits;
        const int t_a = min(split * per, tiles.count);
        Shared::walk(lds, g, rows, seq, tiles, t_a, min(t_a + per, tiles.count), first, 0,
                     [&](int r, int c, const f32x4& sum, float top, float l) {
                         store_part<D>(plan, plan.shared_part(s, rows.a, split, rows.row0 + r), c, sum, top, l);
                     });
        return;
    }
    const uint32_t item = blockIdx.x - (SHARED ? shared_items : 0u), rest = item / (uint32_t)plan.chunks;
    const int w = (int)(item - rest * (uint32_t)plan.chunks);
    const int tile = (int)(rest / (uint32_t)s.kv_heads);
    const Chunk chunk = chunk_at(s, plan, w, lane);
    if (chunk.b < 0) return;
    Rows rows;
    rows.a = (int)(rest - (uint32_t)tile * s.kv_heads);
    rows.b = chunk.b;
    rows.row0 = tile * 16 * OWN;
    rows.n = min(16 * OWN, s.rows - rows.row0);
    const Sequence seq = uniform(sequence(s, chunk.b));
    const int p0 = seq.prefix + seq.kl - seq.ql;
    const int first = p0 + rows.row0 / s.group;
    const int last = p0 + min((rows.row0 + rows.n - 1) / s.group, seq.ql - 1);
    const Tiles<32> tiles(s, seq, first, last, SHARED ? kOwn : kAll);
    const int per = (tiles.count + chunk.chunks - 1) / chunk.chunks;
    const int t_a = min((w - chunk.first) * per, tiles.count);
    const bool direct = !SHARED && chunk.chunks == 1;
    Own::walk(lds, g, rows, seq, tiles, t_a, min(t_a + per, tiles.count), first, last,
              [&](int r, int c, const f32x4& sum, float top, float l) {
                  if (direct) store_row<T, D>(g, row_at(s, rows, seq, r), c, sum, top, l);
                  else store_part<D>(plan, plan.own_part(s, rows.a, w, rows.row0 + r), c, sum, top, l);
              });
}

// The parts of a row in their order, the prefix's first: out = sum 2^(m - M) acc / sum 2^(m - M) l.  A
// workgroup has rows of one sequence; D / 4 lanes have a row, PG groups of them take its parts in turn.
template <typename T, int D, int PG>
__global__ __launch_bounds__(256) void paged_join_kernel(const Args<T> g, uint32_t row_groups)
{
    constexpr int LANES = D / 4, PER = 256 / (LANES * PG);     // rows of a workgroup
    __shared__ f32x4 sum_s[PG][PER * LANES];
    __shared__ float l_s[PG][PER * LANES];
    const Shape& s = g.s;
    const Plan& plan = g.plan;
    const int b = (int)(blockIdx.x / row_groups), tid = threadIdx.x, lane = tid & 63;
    const int at = tid % LANES, slot = tid / LANES % PER, pg = tid / (LANES * PER);
    Chunk chunk = chunks_at(s, plan, b, lane);
    if (!plan.stacked && chunk.chunks == 1) return;            // stored by its workgroup
    const int slice_row = (int)(blockIdx.x % row_groups) * PER + slot;     // (key/value head, row)
    const bool there = slice_row < s.kv_heads * s.rows;
    const int a = there ? slice_row / s.rows : 0, row = there ? slice_row - a * s.rows : 0;
    const int shared = plan.stacked ? plan.shared_splits : 0;
    if (plan.stacked && !plan.scanned) {                       // (a sequence may have nothing of its own)
        const Sequence seq = uniform(sequence(s, b));
        if (units_of(s, plan, seq) == 0) chunk.chunks = 0;
    }
    const int parts = shared + chunk.chunks;
    auto part = [&](int i) -> int64_t {
        return i < shared ? plan.shared_part(s, a, i, b * s.rows + row)
                          : plan.own_part(s, a, chunk.first + i - shared, row);
    };
    float top = kNoRef;
    for (int i = at; i < parts; i += LANES) top = fmaxf(top, plan.ml[part(i)].x);
#pragma unroll
    for (int o = 1; o < LANES; o <<= 1) top = fmaxf(top, __shfl_xor(top, o));
    f32x4 sum = {0.0f, 0.0f, 0.0f, 0.0f};
    float l = 0.0f;
#pragma unroll 4
    for (int i = pg; i < parts; i += PG) {
        const int64_t x = part(i);
        const float2 ml = plan.ml[x];
        const float f = __builtin_amdgcn_exp2f(ml.x - top);
        const f32x4 v = *(const f32x4*)(plan.acc + x * D + 4 * at);
        l = fmaf(f, ml.y, l);
#pragma unroll
        for (int e = 0; e < 4; ++e) sum[e] = fmaf(f, v[e], sum[e]);
    }
    if constexpr (PG > 1) {
        sum_s[pg][slot * LANES + at] = sum;
        l_s[pg][slot * LANES + at] = l;
        __syncthreads();
        if (pg > 0) return;
#pragma unroll
        for (int i = 1; i < PG; ++i) {
            sum += sum_s[i][slot * LANES + at];
            l += l_s[i][slot * LANES + at];
        }
    }
    if (!there) return;
    const Sequence seq = uniform(sequence(s, b));
    store_row<T, D>(g, row_at(s, Rows{row, 1, a, b}, seq, 0), 4 * at, sum, top, l);
}

template <typename T, int D>
hipError_t launch(const Shape& s, const void* q, const void* k, const void* v, void* out, float* lse,
                  void* workspace, hipStream_t stream)
{
    Args<T> g = {(const T*)q, (const T*)k, (const T*)v, (T*)out, lse, s, make_plan(s)};
    Plan& plan = g.plan;
    if (plan.parts) {
        plan.acc = (float*)workspace;
        plan.ml = (float2*)(plan.acc + plan.all_parts(s) * D);
    }
    const int own = tile_rows(s.rows) / 16, shared = plan.stacked ? tile_rows(plan.all_rows) / 16 : 0;
    const uint32_t own_items = (uint32_t)plan.chunks * s.kv_heads * ((s.rows + 16 * own - 1) / (16 * own));
    const uint32_t shared_items =
        shared ? (uint32_t)plan.shared_splits * s.kv_heads * ((plan.all_rows + 16 * shared - 1) / (16 * shared)) : 0u;
    auto kernel = shared == 0   ? own == 1 ? paged_kernel<T, D, 1, 0, 4> : paged_kernel<T, D, 2, 0, 4>
                  : shared == 1 ? paged_kernel<T, D, 1, 1, 4>
                  : own == 1    ? paged_kernel<T, D, 1, 2, 4>
                                : paged_kernel<T, D, 2, 2, 4>;
    kernel<<<own_items + shared_items, 256, 0, stream>>>(g, shared_items);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || !plan.parts) return e;
    const bool many = plan.shared_splits + plan.chunks / s.batch > 8;
    const int per = many ? 256 / (D / 4 * 8) : 256 / (D / 4);
    const uint32_t row_groups = (uint32_t)((s.kv_heads * s.rows + per - 1) / per);
    auto join = many ? paged_join_kernel<T, D, 8> : paged_join_kernel<T, D, 1>;
    join<<<row_groups * (uint32_t)s.batch, 256, 0, stream>>>(g, row_groups);
    return hipGetLastError();
}

}  // namespace paged

size_t paged_fwd_workspace(bool is_bf16, int D, const paged::Shape& s)
{
    const paged::Plan p = paged::make_plan(s);
    return p.parts ? (size_t)p.all_parts(s) * (D + 2) * sizeof(float) : 0;
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
