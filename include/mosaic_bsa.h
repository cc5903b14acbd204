/*
 * mosaic_bsa.h -- C ABI of the MI355X (gfx950) block-sparse attention library.
 *
 * The library implements the hot path of the paper's Block-Sparse Attention
 * (Section "Mosaic", subsection "Block-Sparse Attention") on a row-major
 * lat-lon grid:
 *
 *   - N = H*W tokens are partitioned into m = N/b non-overlapping blocks
 *     (Compression paragraph).  A block is a block_h x block_w tile of the
 *     grid, b = block_h*block_w.  Token t = r*W + c lies in block
 *     beta = (r / block_h)*(W / block_w) + (c / block_w); inside a block,
 *     tokens are ordered row-major, tau = (r % block_h)*block_w + (c % block_w).
 *   - mosaic_bsa_select: mean-pools Q and K per block (pooling equation,
 *     phi = mean), scores every pair of blocks with the pooled dot product
 *     (block-level attention equation; its softmax and 1/sqrt(d_k) are
 *     monotone per row, so they do not change the ranking and are skipped)
 *     and keeps the top-n key blocks of every query block (Selection
 *     paragraph).
 *   - mosaic_bsa_fwd: every token of query block i attends, in one softmax,
 *     to all tokens of block i (Local Attention paragraph) and of the n
 *     selected blocks (fine-grained attention equation).
 *   - mosaic_bsa_bwd: gradients of that attention with the selection held
 *     fixed (Appendix "Block-sparse attention implementation", kernel design).
 *   - mosaic_bsa_fwd_three_branch / mosaic_bsa_bwd_three_branch: the
 *     subsection's own output form, three branches (coarse-grained attention
 *     over the pooled blocks, selection, local attention inside large blocks)
 *     with a softmax each, summed with gate values that the caller supplies
 *     (aggregation equation of the Native Sparse Attention subsection), and
 *     its gradients.
 *   - mosaic_bsa_check_selection, mosaic_bsa_probe_mfma: a checker for
 *     caller-made selections and a measurement aid; neither is on the hot path.
 *
 * Conventions common to all entry points
 *   Pointers  q, k, v, out, dout, dq, dk, dv, sel_idx, lse and the workspace
 *             are DEVICE pointers; `params` is a HOST pointer.  The caller
 *             owns every buffer; the library never allocates, frees or keeps
 *             device memory and never synchronises.  All work is enqueued on
 *             `hip_stream` (a hipStream_t passed as void*, NULL = default
 *             stream); buffers must stay valid until that work has finished.
 *   Layout    q, out, dout, dq: [batch, heads, N, head_dim]; k, v, dk, dv:
 *             [batch, kv_heads, N, head_dim] (kv_heads = heads unless grouped
 *             query attention is asked for); contiguous, head_dim fastest,
 *             element type given by params->dtype, base pointers 16-byte
 *             aligned.
 *             sel_idx: int32 [batch, heads, m, n_select].
 *             lse: fp32 [batch, heads, N], natural-log sum of
 *             exp(softmax_scale * q.k) over the attended keys.
 *   Errors    0 on success, a negative MOSAIC_BSA_ERR_* code otherwise.  All
 *             argument checks run on the host before anything is enqueued;
 *             on error nothing has been launched.  Inputs must be finite.
 *   Masks     by a large finite score (a channel of their own): the forward takes
 *             scores softmax_scale * q.k of any size in fp32 and wherever the
 *             general kernels run (past -2.3e38, where the product with log2(e)
 *             leaves the range of fp32, a key weighs 0, and a row that has no other
 *             key is undefined).  The bf16 kernels for head dims 64 and 128
 *             (blocks of 64 * T tokens, width a power of two; 64, 128 or 256 tokens
 *             at 128) need one score of magnitude below 2^30 among the first 32
 *             attended keys of a row.  Every backward needs one in the row.
 */
#ifndef MOSAIC_BSA_H
#define MOSAIC_BSA_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

enum {
    MOSAIC_BSA_OK = 0,
    MOSAIC_BSA_ERR_NULL = -1,      /* a required pointer is NULL */
    MOSAIC_BSA_ERR_SHAPE = -2,     /* non-positive size, tile does not divide grid, or
                                      kv_heads does not divide heads */
    MOSAIC_BSA_ERR_NSELECT = -3,   /* n_select outside [0, m - 1] ([1, m] in the
                                      three-branch form) */
    MOSAIC_BSA_ERR_HEAD_DIM = -4,  /* head_dim not in {32, 64, 128} */
    MOSAIC_BSA_ERR_DTYPE = -5,     /* dtype not MOSAIC_BSA_F32 / MOSAIC_BSA_BF16 */
    MOSAIC_BSA_ERR_WORKSPACE = -6, /* workspace missing or too small */
    MOSAIC_BSA_ERR_ALIGN = -7,     /* a tensor base pointer is not 16-byte aligned */
    MOSAIC_BSA_ERR_LAUNCH = -8,    /* HIP refused a launch (see hipGetLastError) */
    MOSAIC_BSA_ERR_OP = -9,        /* unknown op for mosaic_bsa_workspace_bytes */
    MOSAIC_BSA_ERR_ROTATION = -10, /* rotation: rotary_dim, axes, layout or scaling */
    MOSAIC_BSA_ERR_STRIDE = -11,   /* a stride that is negative or too large, or rows of an
                                      output that share memory */
    MOSAIC_BSA_ERR_WINDOW = -12    /* window: negative sinks, ring too small for the
                                      window, or a ring in a backward pass */
};

enum { MOSAIC_BSA_F32 = 0, MOSAIC_BSA_BF16 = 1 };
enum { MOSAIC_BSA_OP_SELECT = 0, MOSAIC_BSA_OP_FWD = 1, MOSAIC_BSA_OP_BWD = 2 };

/* Statement of the problem, in the paper's terms. */
typedef struct {
    int32_t batch;          /* B */
    int32_t heads;          /* query heads (key/value heads: kv_heads below) */
    int32_t grid_h, grid_w; /* H, W: lat-lon grid, N = H*W tokens */
    int32_t block_h, block_w; /* tile shape; must divide H and W; b <= 1024 */
    int32_t head_dim;       /* d_k, one of 32, 64, 128 */
    int32_t n_select;       /* n selected blocks per query block, 0 <= n <= m-1 */
    int32_t dtype;          /* element type of q/k/v/out/...: MOSAIC_BSA_F32 or _BF16;
                               accumulation and softmax are fp32 in both cases */
    float softmax_scale;    /* <= 0 selects 1/sqrt(head_dim) (fine-grained
                               attention equation) */
    int32_t kv_heads;       /* key/value heads for grouped query attention (the
                               paper's Attention paragraph: queries attend to a
                               number of shared key-value heads); 0 = heads.
                               Must divide heads: query head a uses key/value
                               head a / (heads / kv_heads).  Selection stays
                               per query head. */
} mosaic_bsa_params;

/* Bytes of device workspace that `op` needs for `params`; 0 if none.
 * Returns 0 as well when params is invalid (the op itself reports why). */
size_t mosaic_bsa_workspace_bytes(const mosaic_bsa_params *params, int op);

/*
 * Block selection (pooling equation, block-level attention equation,
 * Selection paragraph).
 *   q         in   device, [B, heads, N, D]
 *   k         in   device, [B, kv_heads, N, D]
 *   sel_idx   out  device, int32 [B, heads, m, n]: for every query block the
 *                  n key blocks j != i with the largest pooled score, ordered
 *                  by (score descending, block index ascending).
 *   workspace      device scratch of mosaic_bsa_workspace_bytes(.., OP_SELECT)
 *                  bytes; on return it holds the pooled q, fp32
 *                  [B, heads, m, D], at its start and the pooled k, fp32
 *                  [B, kv_heads, m, D], at the byte offset of the pooled
 *                  q's size rounded up to a multiple of 256; the rest is
 *                  scratch.
 * Arithmetic is fixed so that indices are reproducible bit for bit: pooled
 * sums are fp32 adds in in-tile row-major order followed by one multiply by
 * 1/b; a score is the fp32 chain acc = fma(qbar[d], kbar[d], acc), d ascending.
 * n_select == 0 is valid and writes nothing.
 */
int mosaic_bsa_select(const mosaic_bsa_params *params, const void *q, const void *k,
                      int32_t *sel_idx, void *workspace, size_t workspace_bytes,
                      void *hip_stream);

/*
 * mosaic_bsa_select for callers that can neither allocate device memory nor
 * hand over a workspace: code running under HIP graph capture, tight serving
 * loops, harnesses that forbid hipMalloc.  Same arguments, same results (bit
 * for bit) as mosaic_bsa_select, but the selection workspace is a fixed array
 * inside the library, MOSAIC_BSA_STATIC_SCRATCH_BYTES per GPU, that lives from
 * the loading of the library to the end of the process; the call allocates
 * and frees nothing.
 *   - A problem whose selection workspace (mosaic_bsa_workspace_bytes(..,
 *     OP_SELECT)) exceeds MOSAIC_BSA_STATIC_SCRATCH_BYTES is rejected with
 *     MOSAIC_BSA_ERR_WORKSPACE before anything is enqueued.
 *   - All calls on one GPU share that GPU's array: calls whose stream work can
 *     overlap on one GPU race with each other.  Nothing in the array has to
 *     start at zero (every part is written before it is read), so consecutive
 *     calls on one stream need nothing between them.
 *   - The first call on a device looks up the array's address
 *     (hipGetSymbolAddress, with that device current); make it outside graph
 *     capture.  The pooled tensors are not handed back to the caller.
 */
#define MOSAIC_BSA_STATIC_SCRATCH_BYTES (32u << 20)
int mosaic_bsa_select_static(const mosaic_bsa_params *params, const void *q, const void *k,
                             int32_t *sel_idx, void *hip_stream);

/*
 * Block-sparse attention forward (fine-grained attention equation over the
 * union of the query block itself and its selected blocks, one softmax).
 *   q         in   device, [B, heads, N, D]
 *   k, v      in   device, [B, kv_heads, N, D]
 *   sel_idx   in   device, int32 [B, heads, m, n]; every entry in [0, m),
 *                  no duplicates within a row, never the row's own block;
 *                  any order.  Entries are trusted: an out-of-range index is
 *                  undefined behaviour.
 *   out       out  device, [B, heads, N, D], same element type as q; must not
 *                  alias an input.
 *   lse       out  device, fp32 [B, heads, N]; may be NULL.
 *   workspace      unused by this op (may be NULL with workspace_bytes 0).
 * The same call gives the same bits from run to run.  They may differ between calls
 * that hold different numbers of slices: small calls in fp32, and in bf16 where the
 * general kernels run, sum a row's keys in two or four groups (results within the
 * rounding of fp32 sums of each other).
 */
int mosaic_bsa_fwd(const mosaic_bsa_params *params, const void *q, const void *k,
                   const void *v, const int32_t *sel_idx, void *out, float *lse,
                   void *workspace, size_t workspace_bytes, void *hip_stream);

/*
 * Backward of mosaic_bsa_fwd with sel_idx held fixed (no gradient flows
 * through the top-n choice).
 *   q, out, dout        in   device, [B, heads, N, D]
 *   k, v                in   device, [B, kv_heads, N, D]
 *   lse                 in   device, fp32 [B, heads, N] as written by fwd
 *   sel_idx             in   device, same contract as in mosaic_bsa_fwd
 *   dq                  out  device, [B, heads, N, D], element type of q
 *   dk, dv              out  device, [B, kv_heads, N, D] (summed over the query
 *                            heads that share a key/value head)
 *   workspace                device scratch of
 *                            mosaic_bsa_workspace_bytes(.., OP_BWD) bytes; on
 *                            return its start holds delta_l = dout_l . out_l,
 *                            fp32 [B, heads, N] (the rest is scratch: the
 *                            log-sum-exps in base 2 and the reverse map of the
 *                            selection, one bit per (query slice, query
 *                            block, key block)).  dq serves as scratch before it
 *                            is written.
 * Memory that gradients may share with an input, whole tensors only: dq with out
 * (which then is lost), dk with k and dv with v.  Everything else must not overlap.
 * dk/dv of a key block are reduced over the query blocks that attend to it in
 * a fixed order (no floating-point atomics): the same call gives the same bits from run
 * to run.  They may differ between calls that hold different numbers of slices (batch
 * or heads): in small calls two or four groups of wavefronts each sum a part of that
 * order (dk and dv in every type; dq where the general kernels run), and the parts are
 * added in the order of the groups.  Results are within the rounding of fp32 sums of
 * each other.
 */
int mosaic_bsa_bwd(const mosaic_bsa_params *params, const void *q, const void *k,
                   const void *v, const void *out, const float *lse, const void *dout,
                   const int32_t *sel_idx, void *dq, void *dk, void *dv,
                   void *workspace, size_t workspace_bytes, void *hip_stream);

/*
 * The paper's three-branch output (Block-Sparse Attention subsection:
 * Compression, Selection and Local Attention paragraphs; gated sum of the
 * aggregation equation in the Native Sparse Attention subsection):
 *
 *   o_l = g_cg(l) * o_cg(l) + g_fg(l) * o_fg(l) + g_loc(l) * o_loc(l)
 *
 *   coarse     o_cg(l) = sum_j abar_ij vbar_j for every token l of block i,
 *              abar_i = softmax over ALL m blocks of qbar_i . kbar_j * scale,
 *              vbar_j the mean-pooled values;
 *   selection  S_i = the n largest entries of row i over all m blocks (the
 *              block itself is a candidate; 1 <= n_select <= m; ranked by the
 *              pinned fp32 pooled dot product, ties to the smaller index);
 *              o_fg = one softmax over the tokens of the blocks in S_i only;
 *   local      one softmax over the tokens of the large block that contains
 *              l: the aligned group of local_h x local_w mesh tiles
 *              (local_h divides grid_h / block_h, local_w divides
 *              grid_w / block_w; 1 x 1 = the tile itself);
 *   gates      caller-supplied values, one per token, head and branch.
 *
 *   q             in   device, [B, heads, N, D]
 *   k, v          in   device, [B, kv_heads, N, D]
 *   gates         in   device, fp32 [B, heads, N, 3] in the order (coarse,
 *                      selection, local)
 *   out           out  device, [B, heads, N, D], element type of q
 *   sel_idx       out  device, int32 [B, heads, m, n]: S_i in ranking order
 *   workspace          device scratch of
 *                      mosaic_bsa_three_branch_workspace_bytes(..) bytes (pooled
 *                      tensors, block lists, the two attention branches'
 *                      outputs in the element type of q and their
 *                      log-sum-exps); on return it holds what
 *                      mosaic_bsa_bwd_three_branch needs from the forward.
 * The branch outputs are rounded to the element type of q before the gated
 * sum, which runs in fp32.  Bits may differ between calls that hold different numbers
 * of slices, as in mosaic_bsa_fwd.  Errors as for the other entry points; a local
 * group that does not divide the grid of tiles is MOSAIC_BSA_ERR_SHAPE.
 * mosaic_bsa_three_branch_workspace_bytes returns 0 for invalid arguments.
 */
size_t mosaic_bsa_three_branch_workspace_bytes(const mosaic_bsa_params *params,
                                               int32_t local_h, int32_t local_w);
int mosaic_bsa_fwd_three_branch(const mosaic_bsa_params *params, int32_t local_h,
                                int32_t local_w, const void *q, const void *k,
                                const void *v, const float *gates, void *out,
                                int32_t *sel_idx, void *workspace, size_t workspace_bytes,
                                void *hip_stream);

/*
 * Backward of mosaic_bsa_fwd_three_branch with sel_idx held fixed: no gradient
 * flows through the top-n choice; the coarse branch's block softmax, the mean
 * pooling and the gates are differentiated.
 *   q, k, v, gates   in   device, as in the forward
 *   dout             in   device, [B, heads, N, D], element type of q
 *   sel_idx          in   device, as written by the forward
 *   fwd_workspace    in   device, the forward's workspace after the forward
 *                         call on the same inputs, contents intact
 *   dq               out  device, [B, heads, N, D], element type of q
 *   dk, dv           out  device, [B, kv_heads, N, D]
 *   dgates           out  device, fp32 [B, heads, N, 3]: dout . branch output
 *   workspace             device scratch of
 *                         mosaic_bsa_three_branch_bwd_workspace_bytes(..) bytes
 * The upstream gradients of the two attention branches (gate * dout) and the
 * branches' partial gradients are rounded to the element type of q; every sum
 * runs in a fixed order (no floating-point atomics).  Bits may differ between calls
 * that hold different numbers of slices, as in mosaic_bsa_bwd.
 */
size_t mosaic_bsa_three_branch_bwd_workspace_bytes(const mosaic_bsa_params *params,
                                                   int32_t local_h, int32_t local_w);
int mosaic_bsa_bwd_three_branch(const mosaic_bsa_params *params, int32_t local_h,
                                int32_t local_w, const void *q, const void *k,
                                const void *v, const float *gates, const void *dout,
                                const int32_t *sel_idx, const void *fwd_workspace,
                                void *dq, void *dk, void *dv, float *dgates,
                                void *workspace, size_t workspace_bytes, void *hip_stream);

/*
 * ---------------------------------------------------------------------------
 * What sits next to the attention: the rotation of queries and keys by their
 * positions, their norms, and attention inside a sliding window.
 *
 * Tensors of these entry points are [batch, heads, tokens, head_dim] with any
 * strides of the first three dimensions (channels are consecutive), so that q, k
 * and v may be parts of one projection's output [batch, tokens, heads, head_dim]
 * and gradients may be written into such a tensor.  Everything else is as above:
 * device pointers, caller-owned buffers, the caller's stream, checks on the host
 * before anything is enqueued.
 * ---------------------------------------------------------------------------
 */
/* Strides in elements.  token == 0: a contiguous [batch, heads, tokens, head_dim]
 * tensor (batch and head are then ignored).  batch or head may be 0 in an input
 * that is shared by all of them.  Rows of an output must not share memory: each of its
 * strides steps over all that the dimensions with smaller strides reach. */
typedef struct {
    int64_t batch, head, token;
} mosaic_bsa_strides;

enum { MOSAIC_BSA_ROTATE_HALVES = 0, MOSAIC_BSA_ROTATE_PAIRS = 1 };
enum {
    MOSAIC_BSA_SCALE_NONE = 0,
    MOSAIC_BSA_SCALE_LINEAR = 1,   /* every frequency divided by factor */
    MOSAIC_BSA_SCALE_BASE = 2,     /* theta * factor^(d / (d - 2)): the lowest frequency
                                      divided by factor, the highest kept */
    MOSAIC_BSA_SCALE_RAMP = 3      /* by parts (YaRN, Peng et al. 2023): with r = original_tokens
                                      * frequency / 2 pi turns over the trained length,
                                      frequencies with r >= beta_fast are kept, with r <=
                                      beta_slow divided by factor, in between linearly; the
                                      rotated channels are multiplied by 0.1 ln(factor) + 1 */
};
#define MOSAIC_BSA_MAX_PAIRS 64

/* A rotation, in host memory, filled by mosaic_bsa_rotation_init and not changed by
 * any call.  Channels 0 .. rotary_dim - 1 are rotated, the others pass.  They belong to
 * `axes` coordinates (1, or 2 for rows and columns of a grid) in that order, d =
 * rotary_dim / axes channels each; pair i of an axis turns by position * theta^(-2 i / d)
 * (stretched as above) and is made of channels (i, i + d/2) of the axis (HALVES) or
 * (2 i, 2 i + 1) (PAIRS):
 *   (a, b) -> magnitude * (a cos - b sin, b cos + a sin)
 * Frequencies are kept as turns per position in units of 2^-64, so that any 32-bit
 * position gives its angle to 2^-31 turns (frequencies up to 1 radian per position). */
typedef struct {
    int32_t rotary_dim, axes, layout;
    float magnitude;
    uint64_t turns[MOSAIC_BSA_MAX_PAIRS];
} mosaic_bsa_rotation;

/*
 * Fills *out.  rotary_dim: 0 .. 128, a multiple of 2 * axes.  theta > 0 (10000 in the
 * paper).  scaling: MOSAIC_BSA_SCALE_*; factor >= 1; original_tokens > 0 and beta_fast >
 * beta_slow > 0 for RAMP (0, 0: 32 and 1).  inv_freq: NULL, or d / 2 frequencies in radians
 * per position that replace theta and the scaling (out->magnitude is 1 then; the caller may
 * set it to what belongs to those frequencies).
 */
int mosaic_bsa_rotation_init(int32_t rotary_dim, int32_t axes, int32_t layout, double theta,
                             int32_t scaling, double factor, double original_tokens,
                             double beta_fast, double beta_slow, const double *inv_freq,
                             mosaic_bsa_rotation *out);

typedef struct {
    int32_t batch, tokens;     /* B, N */
    int32_t heads, kv_heads;   /* heads of q, and of k and v (0 = heads) */
    int32_t head_dim;          /* 32, 64 or 128 */
    int32_t dtype;             /* MOSAIC_BSA_F32 or _BF16 */
    int32_t cache_tokens;      /* rows of k_out and v_out when `rows` is given */
    int32_t position_batch;    /* int32 values from one batch entry's positions to the
                                  next's; 0: all share [N, axes] */
    float norm_eps;            /* norm forms: added to the mean square; >= 0 (0: a row of
                                  zeros has no norm and gives NaN) */
    mosaic_bsa_strides q, k, v, q_out, k_out, v_out;
} mosaic_bsa_heads_params;

/*
 * Rotation of q and k by their positions, q_out = R q, k_out = R k.
 *   positions  in   device, int32 [N, axes] or [B, N, axes]; NULL (axes 1): 0 .. N - 1
 *   q, k, v    in   device; k and k_out may both be NULL, and so may v and v_out
 *   rows       in   device, int32 [B, N], or NULL.  Given: token n of batch entry b goes to
 *                   row rows[b, n] of k_out and v_out, [B, kv_heads, cache_tokens, D] (a
 *                   key/value cache); a row outside [0, cache_tokens) is not written.
 *                   Two tokens of one entry must not name the same row.
 *   q_out, k_out    out  device; may be q and k (same strides)
 *   v_out           out  device: v as it is
 * Base pointers and strides need the element's alignment only; 16 bytes are fastest.
 * Sums and products run in fp32; the result is rounded once.
 */
int mosaic_bsa_rope_fwd(const mosaic_bsa_heads_params *params, const mosaic_bsa_rotation *rotation,
                        const int32_t *positions, const void *q, const void *k, const void *v,
                        const int32_t *rows, void *q_out, void *k_out, void *v_out,
                        void *hip_stream);
/*
 * Gradient of mosaic_bsa_rope_fwd (without rows and v): dq = R^T dq_out, dk = R^T dk_out.
 * params->q, k: strides of dq, dk; q_out, k_out: strides of dq_out, dk_out.  dq may be dq_out,
 * dk may be dk_out (same strides).
 */
int mosaic_bsa_rope_bwd(const mosaic_bsa_heads_params *params, const mosaic_bsa_rotation *rotation,
                        const int32_t *positions, const void *dq_out, const void *dk_out, void *dq,
                        void *dk, void *hip_stream);
/*
 * Root-mean-square norm of every query and key head and the rotation in one pass:
 *   q_out = R (q_weight * q / sqrt(mean(q^2) + norm_eps)), k likewise with k_weight.
 *   q_weight, k_weight  in  device, fp32 [D]
 * Otherwise as mosaic_bsa_rope_fwd.
 */
int mosaic_bsa_qk_norm_rope_fwd(const mosaic_bsa_heads_params *params,
                                const mosaic_bsa_rotation *rotation, const int32_t *positions,
                                const void *q, const void *k, const void *v,
                                const float *q_weight, const float *k_weight, const int32_t *rows,
                                void *q_out, void *k_out, void *v_out, void *hip_stream);
/*
 * Its gradient (without rows and v).  The sums of dq_weight and dk_weight run in fp32 inside a
 * workgroup, in 64 bits over the workgroups.
 *   q, k                  in   device, the forward's inputs (params->q, k)
 *   dq_out, dk_out        in   device (params->q_out, k_out)
 *   dq, dk                out  device, strides dq_strides, dk_strides; may be dq_out and dk_out, or
 *                              q and k, with the same strides
 *   dq_weight, dk_weight  out  device, fp32 [D], summed over all rows in a fixed order
 *   workspace                  device scratch of mosaic_bsa_qk_norm_rope_workspace_bytes(..) bytes
 * dk_out and dk may both be NULL (k, k_weight, dk_weight are then not read or written).
 */
size_t mosaic_bsa_qk_norm_rope_workspace_bytes(const mosaic_bsa_heads_params *params);
int mosaic_bsa_qk_norm_rope_bwd(const mosaic_bsa_heads_params *params,
                                const mosaic_bsa_rotation *rotation, const int32_t *positions,
                                const void *q, const void *k, const float *q_weight,
                                const float *k_weight, const void *dq_out, const void *dk_out,
                                const mosaic_bsa_strides *dq_strides,
                                const mosaic_bsa_strides *dk_strides, void *dq, void *dk,
                                float *dq_weight, float *dk_weight, void *workspace,
                                size_t workspace_bytes, void *hip_stream);

/*
 * Attention inside a sliding window, with first tokens that stay visible.
 *
 * Sequence b has k_lens[b] keys (token j of it is row j of k and v) and q_lens[b] queries,
 * which stand at its end: query i is at position p = k_lens[b] - q_lens[b] + i.  It sees key j
 * where
 *   0 <= j < k_lens[b]  and  j <= p + window_right  and  (j >= p - window_left or j < n_sink)
 * (a negative window_left or window_right: no bound on that side; window_right = 0 is causal).
 * A query that sees no key, and the rows i >= q_lens[b], give zeros and a log-sum-exp of
 * -infinity; their gradients are zeros, as are those of keys that no query sees.
 *
 * Sizes: with g = heads / kv_heads, fewer than 2^22 slices (batch x kv_heads), 2^29 keys and
 * 2^29 rows (q_tokens x g) of a slice, and 2^24 tiles of 128 rows in all slices together;
 * in the backward also 2^24 tiles of 128 keys and 2^23 groups of 32 sinks; q_tokens below
 * 2^28 on a ring.
 */
typedef struct {
    int32_t batch, heads, kv_heads;    /* kv_heads: 0 = heads; divides heads */
    int32_t q_tokens, k_tokens;        /* rows of q and out; of k and v */
    int32_t head_dim;                  /* 32, 64 or 128 */
    int32_t dtype;                     /* MOSAIC_BSA_F32 or _BF16 */
    int32_t window_left, window_right;
    int32_t n_sink;                    /* first tokens that stay visible */
    int32_t ring;                      /* 0, or forward only: k and v are a ring cache of
                                          k_tokens = n_sink + ring rows; token j < n_sink is row
                                          j, token j >= n_sink row n_sink + (j - n_sink) % ring,
                                          where the newest token with that row is held.
                                          k_lens is required and may exceed k_tokens;
                                          0 <= window_left <= ring - q_tokens */
    float softmax_scale;               /* <= 0 selects 1/sqrt(head_dim) */
    mosaic_bsa_strides q, k, v, out, dout, dq, dk, dv;
} mosaic_bsa_window_params;

/* Bytes of workspace for op MOSAIC_BSA_OP_FWD or _BWD; 0 if none or params is invalid.  Forward: up to
 * 34 MB.  Backward: 8 bytes per query head and token; up to 2 MB x head_dim where few workgroups have
 * long walks; sums of the sinks' keys. */
size_t mosaic_bsa_window_workspace_bytes(const mosaic_bsa_window_params *params, int op);

/*
 *   q, k, v          in   device; bases and strides multiples of 16 bytes
 *   q_lens, k_lens   in   device, int32 [batch], or NULL: q_tokens, k_tokens.  Values are held
 *                         to [0, q_tokens] and [0, k_tokens] (k_lens with a ring: [0, 3 * 2^29])
 *   out              out  device, must not alias an input
 *   lse              out  device, fp32 [batch, heads, q_tokens], natural log; may be NULL
 *   workspace             mosaic_bsa_window_workspace_bytes(.., OP_FWD) bytes (may be 0)
 * Rows of k and v that no query of the call sees may hold anything; everything else must be
 * finite.  Single tokens and short chunks split the keys over workgroups and join the parts
 * in a fixed order: the same call gives the same bits.
 */
int mosaic_bsa_window_fwd(const mosaic_bsa_window_params *params, const void *q, const void *k,
                          const void *v, const int32_t *q_lens, const int32_t *k_lens, void *out,
                          float *lse, void *workspace, size_t workspace_bytes, void *hip_stream);
/*
 *   out, lse         in   device, as written by the forward
 *   dout             in   device
 *   dq, dk, dv       out  device (dk, dv summed over the query heads that share a key/value
 *                         head), must not alias an input or each other
 *   workspace             mosaic_bsa_window_workspace_bytes(.., OP_BWD) bytes
 * Every sum runs in a fixed order (no floating-point atomics).
 */
int mosaic_bsa_window_bwd(const mosaic_bsa_window_params *params, const void *q, const void *k,
                          const void *v, const void *out, const float *lse, const void *dout,
                          const int32_t *q_lens, const int32_t *k_lens, void *dq, void *dk,
                          void *dv, void *workspace, size_t workspace_bytes, void *hip_stream);

/*
 * Checker for selections that were not produced by mosaic_bsa_select: the
 * attention entry points trust sel_idx (an out-of-range index is undefined
 * behaviour), so a caller that builds its own lists can have them counted
 * first.  Not part of the hot path.
 *   sel_idx             in   device, int32 [B, heads, m, n]
 *   own_block_allowed        0: the contract of mosaic_bsa_fwd / _bwd (a row
 *                            never names its own block, n <= m - 1); non-zero:
 *                            the three-branch form's lists (it may, n <= m)
 *   n_bad               out  device, one int32: the number of entries that are
 *                            outside [0, m), repeat an earlier entry of their
 *                            row, or name the own block when that is not
 *                            allowed; 0 means the lists are safe to use.
 */
int mosaic_bsa_check_selection(const mosaic_bsa_params *params, const int32_t *sel_idx,
                               int32_t own_block_allowed, int32_t *n_bad, void *hip_stream);

/*
 * Measurement aid, not part of the attention path: a register-resident bf16
 * matrix-core loop (no loads, no LDS, no vector work) whose rate is the most
 * the matrix pipe sustains on the device at hand.  `workgroups` workgroups of
 * 4 wavefronts each issue 16 * iters 32x32x16 bf16 MFMAs, i.e.
 * workgroups * 4 * 16 * iters * 32768 flop in total; the caller times it.
 *   sink   out  device, workgroups * 256 floats (keeps the loop alive)
 */
int mosaic_bsa_probe_mfma(float *sink, int32_t workgroups, int32_t iters, void *hip_stream);

/* Static, human-readable text for a return code. */
const char *mosaic_bsa_strerror(int code);

#ifdef __cplusplus
}
#endif
#endif /* MOSAIC_BSA_H */
