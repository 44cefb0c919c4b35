/*
 * mmtrain operators around a block's products: rotary positions, the join of a block's branch with the residual stream,
 * the end of a training step (global gradient norm, clipping, the optimizer step that clips as it reads), the embedding that a
 * pack starts with, per-head norms of queries and keys with their rotation, and attention to encoder states of another length.
 *
 * With mmtrain_gemm, mmtrain_attn_fwd / _bwd and mmtrain_adam_step these make up the attention half of a block that differs from
 * the two layers of mmtrain_layer_fwd / _bwd -- another norm placement, gates, other positions -- and the norms and gates around
 * its MLP; the activation inside an MLP (SwiGLU, GELU) is no call of its own.  Conventions (device pointers, caller-owned
 * memory, 16-byte alignment, 256-byte alignment of workspaces, validation on the host before any HIP call, no
 * synchronisation, no allocation, status codes) are those of mmtrain.h.  The current device has to be the one that the
 * pointers belong to.  Sums have a fixed order: a call repeats bit for bit.  All calls may be captured into a HIP graph;
 * two graphs, or two streams, that may run at the same time need a workspace (and a result) each.
 */
#ifndef MMTRAIN_OPS_H
#define MMTRAIN_OPS_H

#include "mmtrain.h"

#ifdef __cplusplus
extern "C" {
#endif

/* ------------------------------------------------------------------------
 * Rotary positions.  Of each head's head_dim features the first rot_dim are rotated in pairs, the others pass through:
 *     a' = m (a cos(p theta_i) - b sin(p theta_i)),   b' = m (b cos(p theta_i) + a sin(p theta_i)),   0 <= i < rot_dim / 2
 * HALF pairs feature i with i + rot_dim / 2, INTERLEAVED feature 2 i with 2 i + 1.  p is the token's position, m the
 * magnitude.  theta_i = base^(-2 i / rot_dim), scaled for contexts longer than the one that the model was trained on:
 *     PLAIN       theta_i
 *     LINEAR      theta_i / factor
 *     WAVELENGTH  theta_i (w_i + (1 - w_i) / factor),  w_i = clamp((n_i - low) / (high - low), 0, 1), where n_i = orig_context
 *                 theta_i / (2 pi) counts the turns of pair i in the trained context: pairs that turn more than `high` times keep
 *                 their frequency, pairs that turn less than `low` times are stretched
 *     RAMP        the same with w_i = 1 - clamp((i - i_high) / (i_low - i_high), 0, 1), linear in the pair's index: i_high and i_low
 *                 are the (real) indices at which a pair would turn `high` and `low` times, rounded down and up and limited to
 *                 0 .. rot_dim - 1 (a difference below 0.001 counts as 0.001)
 * Angles are formed in fp64 and reduced to one turn before they are rounded; products in fp32, one rounding at the end.
 * ------------------------------------------------------------------------ */
typedef enum { MMTRAIN_ROPE_HALF = 0, MMTRAIN_ROPE_INTERLEAVED = 1 } mmtrain_rope_layout;
typedef enum { MMTRAIN_ROPE_PLAIN = 0, MMTRAIN_ROPE_LINEAR = 1, MMTRAIN_ROPE_WAVELENGTH = 2, MMTRAIN_ROPE_RAMP = 3 } mmtrain_rope_scaling;

typedef struct {
    uint32_t struct_size;           /* sizeof(mmtrain_rope_desc) */
    int32_t dtype;                  /* mmtrain_dtype of x and y */
    int32_t n_heads;                /* heads that are rotated, 1 .. 65536 */
    int32_t head_dim;               /* 2 .. 256 */
    int32_t rot_dim;                /* even, 2 .. head_dim (an odd one, or more heads or features: MMTRAIN_ERR_UNSUPPORTED) */
    int32_t layout;                 /* mmtrain_rope_layout */
    int32_t scaling;                /* mmtrain_rope_scaling */
    float base;                     /* > 1 */
    float factor;                   /* >= 1; not read by PLAIN */
    float low, high;                /* turns, 0 < low < high; read by WAVELENGTH and RAMP */
    float orig_context;             /* tokens, > 0; read by WAVELENGTH and RAMP */
    float magnitude;                /* m; 0 => 1, with RAMP 0.1 ln(factor) + 1 */
} mmtrain_rope_desc;

#define MMTRAIN_ROPE_GRADIENT 1u    /* y = the gradient of x for x = the gradient of y: the transposed rotation, times m */

/* y = x with its positions applied.  Row t of x is n_heads * head_dim features at x + t * ld_x elements (the q heads then the
 * k heads of a packed qkv row, say), row t of y at y + t * ld_y; strides in elements, at least n_heads * head_dim.  y may be x
 * (with ld_y = ld_x): then only the rotated features are touched.  Otherwise no element of y may be one of x.
 * Positions: either `batch` (total_tokens = n_tokens; positions restart at 0 in every segment; its masks are not read) or
 * `positions_dev` (device int32 [n_tokens], any values), the other NULL: one token each of many sequences is a call with
 * positions.  Any n_heads, strides and even rot_dim are taken; accesses are 16 bytes wide where head_dim, rot_dim / 2 and the
 * strides are multiples of 8 (bf16) or 4 (fp32) elements, narrower elsewhere. */
MMTRAIN_API int mmtrain_rope(const mmtrain_rope_desc *desc, int32_t n_tokens, const mmtrain_batch *batch,
                             const int32_t *positions_dev, const void *x, int64_t ld_x, void *y, int64_t ld_y, uint32_t flags,
                             void *hip_stream);

/* ------------------------------------------------------------------------
 * The join of a block's branch with the residual stream: the norm behind the block, its gate, the residual's and the branch's
 * scale, and the norm in front of the next block, in one pass:
 *     n = norm_post(branch);   y = residual_scale x + branch_scale gate n;   h = norm_pre(y)
 * RMS: v rsqrt(mean(v^2) + eps) w.  LAYER: (v - mean(v)) rsqrt(var(v) + eps) w + b.  NONE: v.
 * gate: NONE (1), CHANNEL ([hidden]: a learned scale of the branch) or SEGMENT ([n_segments, hidden]: row s for the tokens of
 * segment s of `batch`, for blocks that are conditioned on their sample).
 * Without a branch (branch and y NULL, post_norm and gate NONE) h = norm_pre(x): the norm in front of the first block.
 * h is computed from y before y is rounded to the storage type.  Means and reciprocal deviations ([n_tokens] fp32 each) are
 * kept for the backward pass, which reads y, branch and them.
 * Supported: hidden a multiple of 8, at most 8192, at most 2^30 tokens, and at most 2^20 segments with a SEGMENT gate; anything else:
 * MMTRAIN_ERR_UNSUPPORTED.
 * ------------------------------------------------------------------------ */
typedef enum { MMTRAIN_NORM_NONE = 0, MMTRAIN_NORM_RMS = 1, MMTRAIN_NORM_LAYER = 2 } mmtrain_norm_kind;
typedef enum { MMTRAIN_GATE_NONE = 0, MMTRAIN_GATE_CHANNEL = 1, MMTRAIN_GATE_SEGMENT = 2 } mmtrain_gate_kind;

typedef struct {
    uint32_t struct_size;           /* sizeof(mmtrain_residual_norm_desc) */
    int32_t dtype;                  /* mmtrain_dtype of activations, parameters and (by default) gradients */
    int32_t hidden;
    int32_t post_norm, pre_norm;    /* mmtrain_norm_kind */
    int32_t gate;                   /* mmtrain_gate_kind */
    float post_eps, pre_eps;        /* > 0 where the norm is used */
    float residual_scale, branch_scale;
} mmtrain_residual_norm_desc;

/* Gains and biases [hidden], required where the norm has them (biases: LAYER), NULL elsewhere. */
typedef struct { const void *post_w, *post_b, *gate, *pre_w, *pre_b; } mmtrain_residual_norm_weights;
/* Where to write parameter gradients; NULL: not computed. */
typedef struct { void *post_w, *post_b, *gate, *pre_w, *pre_b; } mmtrain_residual_norm_grads;
/* [n_tokens] fp32 each; means only for LAYER.  Forward writes those that are not NULL, backward needs those of its norms. */
typedef struct { float *post_mean, *post_rstd, *pre_mean, *pre_rstd; } mmtrain_residual_norm_stats;

/* Bytes of `workspace` for backward.  0 on an invalid description.  Never falls as n_tokens grows. */
MMTRAIN_API size_t mmtrain_residual_norm_workspace_bytes(const mmtrain_residual_norm_desc *desc, int32_t n_tokens);

/* Writes y (branch given) and h (pre_norm not NONE; NULL otherwise).  y may be x; no other two of x, branch, y and h may
 * share memory.  `batch` is read with a SEGMENT gate only, `stats` may be NULL. */
MMTRAIN_API int mmtrain_residual_norm_fwd(const mmtrain_residual_norm_desc *desc, int32_t n_tokens, const mmtrain_batch *batch,
                                          const mmtrain_residual_norm_weights *weights, const void *x, const void *branch,
                                          void *y, void *h, const mmtrain_residual_norm_stats *stats, void *hip_stream);

/* From dy (the gradient that reaches y past the next block; NULL: none) and dh (pre_norm not NONE; NULL otherwise) writes
 * dx, d_branch (either may be NULL: not computed) and every non-NULL member of grads (which may be NULL).  `branch` as in
 * forward (NULL for the form without one, where `y` is what forward had as x).  flags: MMTRAIN_BWD_ACCUMULATE_WGRAD,
 * MMTRAIN_BWD_WGRAD_F32, as for mmtrain_layer_bwd.  dx may be dy's buffer and d_branch dh's; otherwise an output may share
 * memory with nothing.  Parameter gradients are fp32 sums over tokens, rounded once: a summand passes through about
 * n_tokens / (256 r) + 50 additions, r = 8, 6, 4, 3 rows at a time for hidden up to 512, 1024, 1536, 2048 and 1 beyond (sums over
 * 400009 rows of 64, all of one sign, are off by 5 x 2^-24 of their value).  The row of a segment gate's gradient that belongs to an empty segment is zero (or keeps what it has,
 * when gradients are added).  workspace: needed where grads has a member. */
MMTRAIN_API int mmtrain_residual_norm_bwd(const mmtrain_residual_norm_desc *desc, int32_t n_tokens, const mmtrain_batch *batch,
                                          const mmtrain_residual_norm_weights *weights, const void *y, const void *branch,
                                          const mmtrain_residual_norm_stats *stats, const void *dy, const void *dh, void *dx,
                                          void *d_branch, const mmtrain_residual_norm_grads *grads, uint32_t flags,
                                          void *workspace, size_t workspace_bytes, void *hip_stream);

/* ------------------------------------------------------------------------
 * Global gradient norm over many tensors, and clipping.  The norm and the factor stay on the device: nothing waits for the
 * host, and the calls may be captured.
 *     sum_sq = sum over all tensors of g^2 (fp64),   norm = sqrt(sum_sq),   factor = norm > max_norm ? max_norm / norm : 1
 * A norm that is not finite as fp32 gives the factor NaN, which stands for "leave everything as it is": mmtrain_grad_clip then writes
 * the gradients unscaled, mmtrain_adam_step_clipped skips the step.
 * ------------------------------------------------------------------------ */
typedef struct {
    const void *grad;               /* device, [n], 16-byte aligned */
    void *out;                      /* device, [n], 16-byte aligned: where the clipped gradient goes; NULL or grad: in place */
    int64_t n;                      /* 0 .. 2^36 (more: MMTRAIN_ERR_UNSUPPORTED) */
    int32_t dtype, out_dtype;       /* mmtrain_dtype; in place they have to be the same */
} mmtrain_grad_tensor;

typedef struct {                    /* device memory, 16-byte aligned */
    double sum_sq;
    float norm, factor;
} mmtrain_grad_norm_result;

/* add to the sum_sq that `result` holds instead of starting at zero: tensors in several calls, or (with no tensors) the norm
 * and the factor anew after the ranks of a sharded model have added up their sum_sq */
#define MMTRAIN_GRAD_NORM_ADD 1u

/* Bytes of `workspace` for mmtrain_grad_norm over n_tensors tensors (a larger count never needs less). */
MMTRAIN_API size_t mmtrain_grad_norm_workspace_bytes(int32_t n_tensors);

/* `tensors`: HOST array; `out` and `out_dtype` are not read.  max_norm >= 0 (infinity: norm only).  The result does not depend
 * on what the workspace holds. */
MMTRAIN_API int mmtrain_grad_norm(const mmtrain_grad_tensor *tensors, int32_t n_tensors, float max_norm, uint32_t flags,
                                  mmtrain_grad_norm_result *result, void *workspace, size_t workspace_bytes, void *hip_stream);

/* out = grad * result->factor, rounded once to out_dtype.  Memory that a tensor writes may not be another tensor's: a list in
 * which it is (the same tensor twice, say) is MMTRAIN_ERR_INVALID_ARG. */
MMTRAIN_API int mmtrain_grad_clip(const mmtrain_grad_tensor *tensors, int32_t n_tensors, const mmtrain_grad_norm_result *result,
                                  void *hip_stream);

/* mmtrain_adam_step with grad * (grad_scale * result->factor) in the place of grad * grad_scale: clipping without another
 * pass over the gradients.  max_norm then applies to the gradients as they are stored, before grad_scale.  Factor NaN: master,
 * the moments and param_out stay as they are (zero_grad still clears the gradient). */
MMTRAIN_API int mmtrain_adam_step_clipped(const mmtrain_adam_desc *desc, int64_t n, float *master, float *grad, float *exp_avg,
                                          float *exp_avg_sq, void *param_out, int32_t param_dtype,
                                          const mmtrain_grad_norm_result *result, void *hip_stream);

/* ------------------------------------------------------------------------
 * Embedding of a multimodal pack.  ids_dev (device int32 [n_tokens]) names the row that each token of the pack starts from:
 *     0 <= id < vocab:            y_t = scale table[id]             (text)
 *     -n_features <= id < 0:      y_t = features[-1 - id]           (an encoder's output row, at its place in the pack)
 *     anything else:              y_t = 0, and no gradient          (padding; vocab itself, say)
 * Backward: d_table[v] = scale times the sum of dy_t over the tokens with id v, d_features[f] the sum over those with id -1 - f.
 * The tokens are sorted by id; a row's sum has a fixed order.
 * Supported: hidden a multiple of 8 up to 65536, vocab >= 1, vocab + n_features <= 2^30, at most 2^30 tokens; anything else:
 * MMTRAIN_ERR_UNSUPPORTED.
 * ------------------------------------------------------------------------ */
typedef struct {
    uint32_t struct_size;           /* sizeof(mmtrain_embed_desc) */
    int32_t dtype;                  /* mmtrain_dtype of table, features, activations and (by default) the table's gradient */
    int32_t hidden;
    int32_t vocab;                  /* rows of the table */
    int32_t n_features;             /* rows of features; 0: none */
    float scale;                    /* of the table's rows (features keep theirs); finite */
} mmtrain_embed_desc;

/* y [n_tokens, hidden] from table [vocab, hidden] and features [n_features, hidden] (NULL where n_features is 0).  y may share
 * memory with nothing. */
MMTRAIN_API int mmtrain_embed_fwd(const mmtrain_embed_desc *desc, int32_t n_tokens, const int32_t *ids_dev, const void *table,
                                  const void *features, void *y, void *hip_stream);

/* Bytes of `workspace` for mmtrain_embed_bwd.  0 on an invalid description.  Never falls as n_tokens grows. */
MMTRAIN_API size_t mmtrain_embed_workspace_bytes(const mmtrain_embed_desc *desc, int32_t n_tokens);

/* From dy [n_tokens, hidden] writes d_table and d_features (either may be NULL: not computed).  flags concern d_table:
 * MMTRAIN_BWD_WGRAD_F32: it is fp32; MMTRAIN_BWD_ACCUMULATE_WGRAD: the sums are added to it, and rows that no token names are not
 * touched; without that flag every row is written, zeros where no token names it.  d_features (the type of `dtype`) is always
 * written as a whole.  Sums are fp32, of chunks of at most 64 + n_tokens / 2048 neighbours in the order
 * and then of the chunks. */
MMTRAIN_API int mmtrain_embed_bwd(const mmtrain_embed_desc *desc, int32_t n_tokens, const int32_t *ids_dev, const void *dy,
                                  void *d_table, void *d_features, uint32_t flags, void *workspace, size_t workspace_bytes,
                                  void *hip_stream);

/* ------------------------------------------------------------------------
 * Norms of queries and keys for each head, and their rotation, in one pass.  A row of x holds n_q_heads query heads, then
 * n_k_heads key heads (what stands behind them, values say, is left alone).  Each head of head_dim features is normalised by itself,
 *     RMS: n = v rsqrt(mean(v^2) + eps) w,   LAYER: n = (v - mean(v)) rsqrt(var(v) + eps) w + b,
 * with one gain (and bias) [head_dim] for all query heads and one for all key heads, and then rotated as mmtrain_rope does it.
 * In front of mmtrain_attn_fwd both kinds are done by one call on the packed qkv; in front of mmtrain_cross_attn_fwd the queries
 * by one (n_k_heads = 0) and the encoder's keys by another (n_q_heads = 0), without a rotation usually.
 * Supported: head_dim a multiple of 8 up to 256, rot_dim a multiple of 4, strides multiples of 8 (bf16) or 4 (fp32) elements, at most
 * 65536 heads and 2^30 tokens; anything else: MMTRAIN_ERR_UNSUPPORTED.
 * ------------------------------------------------------------------------ */
typedef struct {
    uint32_t struct_size;           /* sizeof(mmtrain_qk_norm_desc) */
    int32_t dtype;                  /* mmtrain_dtype of rows, parameters and (by default) parameter gradients */
    int32_t n_q_heads, n_k_heads;   /* either may be 0, not both */
    int32_t head_dim;
    int32_t norm;                   /* MMTRAIN_NORM_RMS or MMTRAIN_NORM_LAYER */
    float eps;                      /* > 0 */
} mmtrain_qk_norm_desc;

/* [head_dim] each, required for heads that there are (biases: LAYER), NULL elsewhere. */
typedef struct { const void *q_w, *q_b, *k_w, *k_b; } mmtrain_qk_norm_weights;
/* Where to write parameter gradients; NULL: not computed. */
typedef struct { void *q_w, *q_b, *k_w, *k_b; } mmtrain_qk_norm_grads;

/* y = the normalised and rotated heads of x; strides as for mmtrain_rope.  `rope` describes the rotation (its dtype and head_dim are
 * desc's, its n_heads n_q_heads + n_k_heads); NULL: none.  Positions as for mmtrain_rope; without a rotation neither `batch` nor
 * positions_dev is read.  y may be x (with ld_y = ld_x), for passes that have no backward pass; otherwise no element of y may be one of x. */
MMTRAIN_API int mmtrain_qk_norm_rope_fwd(const mmtrain_qk_norm_desc *desc, const mmtrain_rope_desc *rope, int32_t n_tokens,
                                         const mmtrain_batch *batch, const int32_t *positions_dev,
                                         const mmtrain_qk_norm_weights *weights, const void *x, int64_t ld_x, void *y, int64_t ld_y,
                                         void *hip_stream);

/* Bytes of `workspace` for backward.  0 on an invalid description.  Never falls as n_tokens grows. */
MMTRAIN_API size_t mmtrain_qk_norm_rope_workspace_bytes(const mmtrain_qk_norm_desc *desc, int32_t n_tokens);

/* From dy (the gradient of y) and forward's x writes dx (NULL: not computed) and every non-NULL member of grads (which may be NULL);
 * statistics are formed anew from x.  dx may be dy's buffer (with ld_dx = ld_dy); otherwise an output may share memory with nothing.
 * flags: MMTRAIN_BWD_ACCUMULATE_WGRAD, MMTRAIN_BWD_WGRAD_F32.  workspace: needed where grads has a member. */
MMTRAIN_API int mmtrain_qk_norm_rope_bwd(const mmtrain_qk_norm_desc *desc, const mmtrain_rope_desc *rope, int32_t n_tokens,
                                         const mmtrain_batch *batch, const int32_t *positions_dev,
                                         const mmtrain_qk_norm_weights *weights, const void *x, int64_t ld_x, const void *dy,
                                         int64_t ld_dy, void *dx, int64_t ld_dx, const mmtrain_qk_norm_grads *grads, uint32_t flags,
                                         void *workspace, size_t workspace_bytes, void *hip_stream);

/* ------------------------------------------------------------------------
 * Cross attention: queries of a pack attend to keys and values of another length (an encoder's states).  The queries are cut into
 * runs; all tokens of run s, cu_q[s] .. cu_q[s + 1] - 1, see the keys kv_begin[s] .. kv_end[s] - 1 and no others:
 *     o_t = sum_j softmax_j(softmax_scale q_t . k_j) v_j,    lse_t = ln sum_j exp(softmax_scale q_t . k_j)
 * A pack whose samples have their own images: kv_begin = cu_kv, kv_end = cu_kv + 1 (the same array).  Runs may see the same keys (several
 * continuations of one prompt) or overlapping ranges (text that sees the images so far).  kv_begin[s] = kv_end[s]: the run sees
 * nothing, o = 0, lse = -infinity, no gradient.  What a query does not see does not reach it, not even an infinity or NaN.
 * Scores, softmax statistics and sums are fp32.  With MMTRAIN_BF16 the operands of all products are bf16, so the probabilities (and, for the gradients, P and dS) are
 * rounded to bf16 before they meet V, dO, K and Q: each is off by half a step, 2^-8 of its value, at most; o by l2 0.0023 of its norm where its own rounding makes
 * 0.0017.  MMTRAIN_F32 rounds nothing to fewer bits.
 * Grouped heads as in mmtrain_layer_desc: query head h reads key/value head h / (n_heads / n_kv_heads).
 * One token for each of many sequences is a call with runs of one token: with few queries the keys are shared out over the chip.
 * Supported: head_dim a multiple of 16 up to 128, n_heads % n_kv_heads = 0, at most 4096 heads, 65536 runs, 2^28 rows of a key/value head (query
 * tokens times the heads that share it), 2^30 key tokens, query tokens and runs together times heads below 2^31, strides multiples of 8 (bf16) or 4 (fp32) elements below
 * 2^24, and fewer than 2^23 - 1 workgroups, counted as q_tokens n_heads / 32 + runs n_kv_heads and as (kv_tokens / 128 + 2 runs + 1) n_kv_heads (fp32: / 16, and / 16
 * and 8 times the runs' part); anything else: MMTRAIN_ERR_UNSUPPORTED.
 * ------------------------------------------------------------------------ */
typedef struct {
    uint32_t struct_size;           /* sizeof(mmtrain_cross_attn_desc) */
    int32_t dtype;                  /* mmtrain_dtype */
    int32_t n_heads, n_kv_heads, head_dim;
    float softmax_scale;            /* > 0; 0 => 1/sqrt(head_dim) */
} mmtrain_cross_attn_desc;

/* The host arrays hold the same values as the device arrays: validation and launch sizing.  A captured call is replayed for the ranges
 * that it was captured with. */
typedef struct {
    int32_t q_tokens, kv_tokens;    /* rows of q, and of k and v */
    int32_t n_segments;             /* runs of queries, S */
    const int32_t *cu_q_dev, *cu_q_host;            /* [S + 1]: 0, non-decreasing, q_tokens */
    const int32_t *kv_begin_dev, *kv_begin_host;    /* [S] */
    const int32_t *kv_end_dev, *kv_end_host;        /* [S]: kv_begin <= kv_end <= kv_tokens */
} mmtrain_cross_batch;

/* Rows of q and o: n_heads heads, of k and v: n_kv_heads heads; strides in elements (k and v may be columns of one tensor). */
typedef struct {
    const void *q; int64_t ld_q;
    const void *k; int64_t ld_k;
    const void *v; int64_t ld_v;
    void *o; int64_t ld_o;          /* written by fwd, read by bwd */
    float *lse;                     /* [n_heads, q_tokens]; fwd: may be NULL; bwd: required */
} mmtrain_cross_attn_tensors;
typedef struct {
    const void *d_o; int64_t ld_do;
    void *d_q; int64_t ld_dq;       /* NULL: not computed */
    void *d_k; int64_t ld_dk;       /* d_k and d_v: both, or neither (a frozen encoder) */
    void *d_v; int64_t ld_dv;
} mmtrain_cross_attn_grads;

/* Bytes of `workspace` for fwd (is_bwd = 0) or bwd (is_bwd = 1); the host arrays of `batch` are read.  0 where the call would be refused. */
MMTRAIN_API size_t mmtrain_cross_attn_workspace_bytes(const mmtrain_cross_attn_desc *desc, const mmtrain_cross_batch *batch, int is_bwd);

MMTRAIN_API int mmtrain_cross_attn_fwd(const mmtrain_cross_attn_desc *desc, const mmtrain_cross_batch *batch,
                                       const mmtrain_cross_attn_tensors *tensors, void *workspace, size_t workspace_bytes, void *hip_stream);

/* Every row of d_q, d_k and d_v is written, zeros for queries that see nothing and keys that nobody sees.  Where d_k and d_v are computed, kv_begin and
 * kv_end have to be non-decreasing over the runs that see something (MMTRAIN_ERR_BAD_SEGMENTS), so that the runs which see a key
 * follow one another.  Outputs may share memory with nothing. */
MMTRAIN_API int mmtrain_cross_attn_bwd(const mmtrain_cross_attn_desc *desc, const mmtrain_cross_batch *batch,
                                       const mmtrain_cross_attn_tensors *tensors, const mmtrain_cross_attn_grads *grads,
                                       void *workspace, size_t workspace_bytes, void *hip_stream);

#ifdef __cplusplus
}
#endif
#endif /* MMTRAIN_OPS_H */
