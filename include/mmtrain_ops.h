/*
 * mmtrain operators around a block's products: rotary positions, the join of a block's branch with the residual stream,
 * and the end of a training step (global gradient norm, clipping, the optimizer step that clips as it reads).
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

#ifdef __cplusplus
}
#endif
#endif /* MMTRAIN_OPS_H */
