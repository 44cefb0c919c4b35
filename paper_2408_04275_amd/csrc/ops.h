// Internal launch interface of the operators in mmtrain_ops.h (see kernels.h for the conventions).
#pragma once
#include "kernels.h"

namespace mmt {

// rope.hip.  turns[i] = frequency of pair i in turns per position.
constexpr int ROPE_MAX_HALF = 128, ROPE_MAX_HEADS = 1 << 16;
struct RopeArgs {
    int T, heads, d, half;          // half = rot_dim / 2
    bool interleaved;
    const int *positions;           // device [T], or null: from cu
    const int *cu; int S;
    const void *x; long ldx;
    void *y; long ldy;
    float cos_scale, sin_scale;     // magnitude, and magnitude with the direction's sign
    double turns[ROPE_MAX_HALF];
};
hipError_t rope(int dtype, const RopeArgs &a, hipStream_t st);

// residual_norm.hip: n = norm_post(b); y = alpha x + beta gate n; h = norm_pre(y)
enum { NORM_NONE = 0, NORM_RMS = 1, NORM_LAYER = 2 };
enum { GATE_NONE = 0, GATE_CHANNEL = 1, GATE_SEGMENT = 2 };
struct JoinArgs {
    int T, H, post, pre, gate;
    float post_eps, pre_eps, alpha, beta;
    const int *cu; int S;           // segment gates
    const void *post_w, *post_b, *gate_v, *pre_w, *pre_b;
    float *post_mean, *post_rstd, *pre_mean, *pre_rstd;
    const void *b;                  // null: no branch
    const void *x;                  // forward; y and h may be null
    void *y, *h;
    const void *dy, *dh;            // backward (y is read); dy, dx, db may be null
    void *dx, *db;
    // backward: partial sums, null where not wanted.  post_w, post_b, pre_w, pre_b and a channel's gate: [join_bwd_blocks][H];
    // a segment's gate: [2 * join_bwd_blocks][H], see there
    float *p_post_w, *p_post_b, *p_gate, *p_pre_w, *p_pre_b;
    void *d_post_w, *d_post_b, *d_gate, *d_pre_w, *d_pre_b;     // the gradients, null where not wanted
    int grad_f32, accumulate;       // their type, and whether they are added to
};
constexpr int JOIN_MAX_ROWS = 1 << 30;          // a row and the next ones' numbers fit an int
constexpr int JOIN_MAX_SEGMENTS = 1 << 20;      // with a segment gate: [segments][H] are the gates alone
hipError_t join_fwd(int dtype, const JoinArgs &a, hipStream_t st);
// workgroups of the backward kernel: never fewer for more rows
int join_bwd_blocks(int T, int H);
hipError_t join_bwd(int dtype, const JoinArgs &a, hipStream_t st);

// grad_norm.hip
constexpr int GRAD_BATCH = 128, GRAD_FEW = 16;      // tensors a launch; at most so many go as a smaller argument
template <int N> struct GradBatch {
    const void *in[N];
    void *out[N];
    long n[N];
    int first[N + 1];               // first chunk of each tensor; [count] = all
    unsigned char in_f32[N], out_f32[N];
    int count, chunk;               // elements a chunk, a multiple of 8
};
constexpr int GRAD_BLOCKS = 2048;   // workgroups, and partial sums, of a launch at most: eight of 256 threads on each compute unit
struct GradResult { double sum_sq; float norm, factor; };
// For GRAD_BATCH and GRAD_FEW.  grad_chunks cuts a batch whose in, out, n, types and count are set into chunks (first, chunk).
template <int N> void grad_chunks(GradBatch<N> &b);
template <int N> int grad_norm_blocks(const GradBatch<N> &b);
template <int N> hipError_t grad_sum_sq(const GradBatch<N> &b, double *part, hipStream_t st);
hipError_t grad_norm_finish(const double *part, int n, float max_norm, bool add, GradResult *result, hipStream_t st);
bool grad_clip_streams(size_t bytes_written);       // by a whole call
template <int N> hipError_t grad_clip(const GradBatch<N> &b, const GradResult *result, bool stream, hipStream_t st);

}  // namespace mmt
