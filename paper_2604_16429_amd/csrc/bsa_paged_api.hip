// Entry points of the attention over a cache in pages: checks on the host, then launches.  The
// contract is in include/mosaic_bsa.h; mosaic_bsa_paged_append is in bsa_heads.hip.
#include <math.h>

#include "bsa_paged.h"

namespace {

struct Checked {
    bsa::paged::Shape s;
    int D;
    bool is_bf16;
};

int check_params(const mosaic_bsa_paged_params* p, Checked* c)
{
    if (!p) return MOSAIC_BSA_ERR_NULL;
    if (p->batch <= 0 || p->heads <= 0 || p->kv_heads < 0 || p->q_tokens <= 0) return MOSAIC_BSA_ERR_SHAPE;
    if (int rc = bsa::check_pages(*p)) return rc;
    if (p->head_dim != 32 && p->head_dim != 64 && p->head_dim != 128) return MOSAIC_BSA_ERR_HEAD_DIM;
    if (p->dtype != MOSAIC_BSA_F32 && p->dtype != MOSAIC_BSA_BF16) return MOSAIC_BSA_ERR_DTYPE;
    if (p->n_sink < 0) return MOSAIC_BSA_ERR_WINDOW;
    c->D = p->head_dim;
    c->is_bf16 = p->dtype == MOSAIC_BSA_BF16;
    bsa::paged::Shape& s = c->s;
    s = {};
    s.batch = p->batch;
    s.heads = p->heads;
    s.kv_heads = p->kv_heads == 0 ? p->heads : p->kv_heads;
    s.group = s.heads / s.kv_heads;
    s.q_tokens = p->q_tokens;
    s.rows = p->q_tokens * s.group;
    s.pages = p->pages;
    s.page_shift = __builtin_ctz((unsigned)p->page_tokens);
    s.table_pages = p->table_pages;
    s.prefix_tokens = p->prefix_tokens;
    s.left = p->window_left < 0 || p->window_left > bsa::paged::kUnbounded ? bsa::paged::kUnbounded
                                                                           : p->window_left;
    s.sinks = p->n_sink;
    s.scale = p->softmax_scale > 0.0f ? p->softmax_scale : 1.0f / sqrtf((float)p->head_dim);
    // launches of less than 2^32 work items: 256 to a tile and, where sums are joined, to 8 rows
    if ((int64_t)s.batch * s.kv_heads * ((s.rows + 31) / 32) >= 1 << 21) return MOSAIC_BSA_ERR_SHAPE;
    return MOSAIC_BSA_OK;
}

// Base pointer and strides of one tensor; the strides, written out, go to *to.
int check_tensor(const Checked& c, const void* ptr, const mosaic_bsa_strides& st, int batch, int heads,
                 int tokens, bool output, mosaic_bsa_strides* to)
{
    if (!ptr) return MOSAIC_BSA_ERR_NULL;
    const int D = c.D, per16 = c.is_bf16 ? 8 : 4;
    if (bsa::bad_strides(st, batch, heads, tokens, D, output)) return MOSAIC_BSA_ERR_STRIDE;
    *to = bsa::strides_of(st, heads, tokens, D);
    if ((uintptr_t)ptr & 15u || to->batch % per16 || to->head % per16 || to->token % per16)
        return MOSAIC_BSA_ERR_ALIGN;
    if (output && bsa::rows_meet(st, batch, heads, tokens, D)) return MOSAIC_BSA_ERR_STRIDE;
    return MOSAIC_BSA_OK;
}

bool unaligned4(const void* p) { return ((uintptr_t)p & 3u) != 0; }

}  // namespace

extern "C" size_t mosaic_bsa_paged_workspace_bytes(const mosaic_bsa_paged_params* params)
{
    Checked c;
    if (check_params(params, &c) != MOSAIC_BSA_OK) return 0;
    return bsa::paged_fwd_workspace(c.is_bf16, c.D, c.s);
}

extern "C" int mosaic_bsa_paged_fwd(const mosaic_bsa_paged_params* params, const void* q,
                                    const void* k_pages, const void* v_pages, const int32_t* q_lens,
                                    const int32_t* k_lens, const int32_t* page_table,
                                    const int32_t* prefix_table, const int32_t* prefix_len, void* out,
                                    float* lse, void* workspace, size_t workspace_bytes,
                                    void* hip_stream)
{
    Checked c;
    if (int rc = check_params(params, &c)) return rc;
    const mosaic_bsa_paged_params& p = *params;
    bsa::paged::Shape& s = c.s;
    if (int rc = check_tensor(c, q, p.q, s.batch, s.heads, s.q_tokens, false, &s.q)) return rc;
    if (int rc = check_tensor(c, k_pages, p.k_pages, s.pages, s.kv_heads, p.page_tokens, false, &s.k))
        return rc;
    if (int rc = check_tensor(c, v_pages, p.v_pages, s.pages, s.kv_heads, p.page_tokens, false, &s.v))
        return rc;
    if (int rc = check_tensor(c, out, p.out, s.batch, s.heads, s.q_tokens, true, &s.out)) return rc;
    if (!k_lens || !page_table || (s.prefix_tokens > 0 && !prefix_table)) return MOSAIC_BSA_ERR_NULL;
    if (unaligned4(lse) || unaligned4(q_lens) || unaligned4(k_lens) || unaligned4(page_table) ||
        unaligned4(prefix_table) || unaligned4(prefix_len) || ((uintptr_t)workspace & 15u))
        return MOSAIC_BSA_ERR_ALIGN;
    const size_t need = bsa::paged_fwd_workspace(c.is_bf16, c.D, s);
    if (need && (!workspace || workspace_bytes < need)) return MOSAIC_BSA_ERR_WORKSPACE;
    s.q_lens = q_lens;
    s.k_lens = k_lens;
    s.table = page_table;
    s.prefix_table = prefix_table;
    s.prefix_len = prefix_len;
    return bsa::launch_paged_fwd(c.is_bf16, c.D, s, q, k_pages, v_pages, out, lse, workspace,
                                 (hipStream_t)hip_stream) == hipSuccess
               ? MOSAIC_BSA_OK
               : MOSAIC_BSA_ERR_LAUNCH;
}
