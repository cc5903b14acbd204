// Entry points of the windowed attention: checks on the host, then launches.  The contract
// is in include/mosaic_bsa.h.
#include <math.h>

#include <algorithm>

#include "bsa_window.h"

namespace {

using bsa::win::kMostRingChunk;
using bsa::win::kUnbounded;
constexpr int32_t kMostTokens = 1 << 29;

struct Checked {
    bsa::win::Shape s;
    int D;
    bool is_bf16;
};

int32_t bound(int32_t x) { return x < 0 || x > kUnbounded ? kUnbounded : x; }

int check_params(const mosaic_bsa_window_params* p, bool backward, Checked* c)
{
    if (!p) return MOSAIC_BSA_ERR_NULL;
    if (p->batch <= 0 || p->heads <= 0 || p->kv_heads < 0 || p->q_tokens <= 0 || p->k_tokens <= 0)
        return MOSAIC_BSA_ERR_SHAPE;
    const int kv_heads = p->kv_heads == 0 ? p->heads : p->kv_heads;
    if (kv_heads > p->heads || p->heads % kv_heads) return MOSAIC_BSA_ERR_SHAPE;
    const int group = p->heads / kv_heads;
    const int64_t rows = (int64_t)p->q_tokens * group;
    const int64_t slices = (int64_t)p->batch * kv_heads;
    // sums of positions and lengths stay below 2^31, launches below 2^32 work items: 256 of them to a tile
    // of 128 rows, up to 1,024 to a slice of few rows
    if (rows >= kMostTokens || p->k_tokens >= kMostTokens || slices >= (int64_t)1 << 22 ||
        slices * ((rows + 127) / 128) >= (int64_t)1 << 24)
        return MOSAIC_BSA_ERR_SHAPE;
    if (p->ring > 0 && p->q_tokens >= kMostRingChunk) return MOSAIC_BSA_ERR_SHAPE;
    // backward: 256 to a tile of 128 keys, 512 to a group of 32 that holds sinks
    if (backward && (slices * (((int64_t)p->k_tokens + 127) / 128) >= (int64_t)1 << 24 ||
                     slices * (((int64_t)std::min(p->n_sink, p->k_tokens) + 31) / 32) >= (int64_t)1 << 23))
        return MOSAIC_BSA_ERR_SHAPE;
    if (p->head_dim != 32 && p->head_dim != 64 && p->head_dim != 128) return MOSAIC_BSA_ERR_HEAD_DIM;
    if (p->dtype != MOSAIC_BSA_F32 && p->dtype != MOSAIC_BSA_BF16) return MOSAIC_BSA_ERR_DTYPE;
    if (p->n_sink < 0 || p->ring < 0) return MOSAIC_BSA_ERR_WINDOW;
    if (p->ring > 0 && ((int64_t)p->n_sink + p->ring != p->k_tokens || p->window_left < 0 ||
                        (int64_t)p->window_left + p->q_tokens > p->ring))
        return MOSAIC_BSA_ERR_WINDOW;
    c->D = p->head_dim;
    c->is_bf16 = p->dtype == MOSAIC_BSA_BF16;
    bsa::win::Shape& s = c->s;
    s.batch = p->batch;
    s.heads = p->heads;
    s.kv_heads = kv_heads;
    s.group = group;
    s.q_tokens = p->q_tokens;
    s.k_tokens = p->k_tokens;
    s.rows = (int32_t)rows;
    s.left = bound(p->window_left);
    // (the queries stand at the end: no key is further to the right of one than the last query)
    s.right = std::min(bound(p->window_right), p->q_tokens);
    s.sinks = p->n_sink < p->k_tokens ? p->n_sink : p->k_tokens;
    s.ring = p->ring;
    s.scale = p->softmax_scale > 0.0f ? p->softmax_scale : 1.0f / sqrtf((float)p->head_dim);
    s.q_lens = s.k_lens = nullptr;
    s.q = s.k = s.v = s.out = s.dout = s.dq = s.dk = s.dv = mosaic_bsa_strides{0, 0, 0};
    return MOSAIC_BSA_OK;
}

// Base pointer and strides of one tensor; the strides, written out, go to *to.
int check_tensor(const Checked& c, const void* ptr, const mosaic_bsa_strides& st, int heads,
                 int tokens, bool output, mosaic_bsa_strides* to)
{
    if (!ptr) return MOSAIC_BSA_ERR_NULL;
    const int D = c.D, per16 = c.is_bf16 ? 8 : 4;
    if (bsa::bad_strides(st, c.s.batch, heads, tokens, D, output))
        return MOSAIC_BSA_ERR_STRIDE;
    *to = bsa::strides_of(st, heads, tokens, D);
    if ((uintptr_t)ptr & 15u || to->batch % per16 || to->head % per16 || to->token % per16)
        return MOSAIC_BSA_ERR_ALIGN;
    if (output && bsa::rows_meet(st, c.s.batch, heads, tokens, D)) return MOSAIC_BSA_ERR_STRIDE;
    return MOSAIC_BSA_OK;
}

bool unaligned4(const void* p) { return ((uintptr_t)p & 3u) != 0; }

}  // namespace

extern "C" size_t mosaic_bsa_window_workspace_bytes(const mosaic_bsa_window_params* params, int op)
{
    Checked c;
    if (check_params(params, op == MOSAIC_BSA_OP_BWD, &c) != MOSAIC_BSA_OK) return 0;
    if (op == MOSAIC_BSA_OP_FWD) return bsa::window_fwd_workspace(c.is_bf16, c.D, c.s);
    if (op == MOSAIC_BSA_OP_BWD && !c.s.ring) return bsa::window_bwd_workspace(c.is_bf16, c.D, c.s);
    return 0;
}

extern "C" int mosaic_bsa_window_fwd(const mosaic_bsa_window_params* params, const void* q,
                                     const void* k, const void* v, const int32_t* q_lens,
                                     const int32_t* k_lens, void* out, float* lse, void* workspace,
                                     size_t workspace_bytes, void* hip_stream)
{
    Checked c;
    if (int rc = check_params(params, false, &c)) return rc;
    const mosaic_bsa_window_params& p = *params;
    bsa::win::Shape& s = c.s;
    if (int rc = check_tensor(c, q, p.q, s.heads, s.q_tokens, false, &s.q)) return rc;
    if (int rc = check_tensor(c, k, p.k, s.kv_heads, s.k_tokens, false, &s.k)) return rc;
    if (int rc = check_tensor(c, v, p.v, s.kv_heads, s.k_tokens, false, &s.v)) return rc;
    if (int rc = check_tensor(c, out, p.out, s.heads, s.q_tokens, true, &s.out)) return rc;
    if (s.ring && !k_lens) return MOSAIC_BSA_ERR_NULL;
    if (unaligned4(lse) || unaligned4(q_lens) || unaligned4(k_lens) || ((uintptr_t)workspace & 15u))
        return MOSAIC_BSA_ERR_ALIGN;
    const size_t need = bsa::window_fwd_workspace(c.is_bf16, c.D, s);
    if (need && (!workspace || workspace_bytes < need)) return MOSAIC_BSA_ERR_WORKSPACE;
    s.q_lens = q_lens;
    s.k_lens = k_lens;
    return bsa::launch_window_fwd(c.is_bf16, c.D, s, q, k, v, out, lse, workspace,
                                  (hipStream_t)hip_stream) == hipSuccess
               ? MOSAIC_BSA_OK
               : MOSAIC_BSA_ERR_LAUNCH;
}

extern "C" int mosaic_bsa_window_bwd(const mosaic_bsa_window_params* params, const void* q,
                                     const void* k, const void* v, const void* out,
                                     const float* lse, const void* dout, const int32_t* q_lens,
                                     const int32_t* k_lens, void* dq, void* dk, void* dv,
                                     void* workspace, size_t workspace_bytes, void* hip_stream)
{
    Checked c;
    if (int rc = check_params(params, true, &c)) return rc;
    const mosaic_bsa_window_params& p = *params;
    bsa::win::Shape& s = c.s;
    if (s.ring) return MOSAIC_BSA_ERR_WINDOW;
    if (int rc = check_tensor(c, q, p.q, s.heads, s.q_tokens, false, &s.q)) return rc;
    if (int rc = check_tensor(c, k, p.k, s.kv_heads, s.k_tokens, false, &s.k)) return rc;
    if (int rc = check_tensor(c, v, p.v, s.kv_heads, s.k_tokens, false, &s.v)) return rc;
    if (int rc = check_tensor(c, out, p.out, s.heads, s.q_tokens, false, &s.out)) return rc;
    if (int rc = check_tensor(c, dout, p.dout, s.heads, s.q_tokens, false, &s.dout)) return rc;
    if (int rc = check_tensor(c, dq, p.dq, s.heads, s.q_tokens, true, &s.dq)) return rc;
    if (int rc = check_tensor(c, dk, p.dk, s.kv_heads, s.k_tokens, true, &s.dk)) return rc;
    if (int rc = check_tensor(c, dv, p.dv, s.kv_heads, s.k_tokens, true, &s.dv)) return rc;
    if (!lse) return MOSAIC_BSA_ERR_NULL;
    if (unaligned4(lse) || unaligned4(q_lens) || unaligned4(k_lens) || ((uintptr_t)workspace & 15u))
        return MOSAIC_BSA_ERR_ALIGN;
    const size_t need = bsa::window_bwd_workspace(c.is_bf16, c.D, s);
    if (!workspace || workspace_bytes < need) return MOSAIC_BSA_ERR_WORKSPACE;
    s.q_lens = q_lens;
    s.k_lens = k_lens;
    return bsa::launch_window_bwd(c.is_bf16, c.D, s, q, k, v, out, lse, dout, dq, dk, dv, workspace,
                                  (hipStream_t)hip_stream) == hipSuccess
               ? MOSAIC_BSA_OK
               : MOSAIC_BSA_ERR_LAUNCH;
}
