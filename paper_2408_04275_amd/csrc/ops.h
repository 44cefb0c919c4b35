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

// qk_norm.hip: per-head norms and rotation
struct QkNormArgs {
    RopeArgs r;                     // rows, heads (queries first), rotation (half = 0: none)
    int nq, norm;                   // query heads; NORM_RMS or NORM_LAYER
    float eps;
    const void *q_w, *q_b, *k_w, *k_b;
    const void *dy; long lddy;      // backward: r.y is dx (may be null)
    float *part[4];                 // partial sums of q_w, q_b, k_w, k_b [qk_norm_bwd_blocks][d], null where not wanted
    void *grad[4];
    int grad_f32, accumulate;
};
constexpr int QK_MAX_ROWS = 1 << 30;
hipError_t qk_norm_fwd(int dtype, const QkNormArgs &a, hipStream_t st);
int qk_norm_bwd_blocks(int T, int norm);        // never fewer for more rows
hipError_t qk_norm_bwd(int dtype, const QkNormArgs &a, hipStream_t st);

// embed.hip
constexpr int EMBED_MAX_ROWS = 1 << 30;
struct EmbedArgs {
    int T, H, vocab, features;
    float scale;
    const int *ids;
    const void *table, *rows;       // forward
    void *y;
    const void *dy;                 // backward
    void *d_table, *d_rows;         // null where not wanted
    int table_f32, accumulate;
    void *ws;
};
hipError_t embed_fwd(int dtype, const EmbedArgs &a, hipStream_t st);
size_t embed_bwd_bytes(int T, int H);
hipError_t embed_bwd(int dtype, const EmbedArgs &a, hipStream_t st);

// cross_plan.hip, cross_mfma.hip, cross_mfma_bwd.hip, cross_f32.hip
constexpr int CROSS_MAX_SEGMENTS = 1 << 16;
struct CrossArgs {
    int Tq, Tk, S, nh, nkv, d;
    float scale;
    const int *cu, *begin, *end;    // device
    const void *q; long ldq;
    const void *k; long ldk;
    const void *v; long ldv;
    void *o; long ldo;
    float *lse;                     // [nh, Tq]; forward: may be null
    const void *d_o; long lddo;     // backward
    void *dq; long lddq;            // null where not wanted
    void *dk; long lddk;
    void *dv; long lddv;
    float *D;                       // backward scratch [nh, Tq]: rowsum(dO * O)
    // Runs that follow one another and see the same keys are worked on as one (within 64 runs from a multiple of 64 on)
    uint8_t order[64], last[64];    // up to 64 runs: first and last of each such sequence, by falling number of keys
    int n_sequences;
    const int *prefix;              // more: first item of each run [S + 1], none of those behind a sequence's first; first run behind its sequence [S]
    int chunk;                      // keys of a workgroup; 0: all of its run's
    float *part; float2 *part_ml;   // partial results of the chunks [item, head][rows][d], their maxima and sums (forward)
    // dK and dV: see make_plan
    int4 *tiles, *steps;
    int n_tiles, n_steps;           // n_tiles 0: not wanted
    int *plan;                      // scratch for many runs
    int parts;                      // workgroups that share the rows which see a tile of keys
    float *dkv_part;                // [parts][Tk][2 nkv d], where there are several
};
// What a call is planned from: sizes, and the runs' host arrays
struct CrossShape { int Tq, Tk, S, nh, nkv, d; const int *cu, *begin, *end; };
struct CrossPlan {
    int rows, chunk, items;         // rows of a workgroup, keys of a chunk (0: not cut), workgroups per key/value head
    int waves;                      // bf16, few rows: wavefronts of a workgroup
    bool table;                     // items are found in a table
};
struct CrossBwdPlan {
    int rows, chunk, items;         // dQ: as above
    bool table, dkv;
    int tiles, steps, parts;        // dK and dV: tiles of keys, tiles of rows of all runs, workgroups per tile of keys
    bool own;                       // ... fp32: a wavefront has 16 keys to itself
};
// Plans, workspaces (256-byte aligned) and calls.  dkv: the gradients of keys and values are wanted
CrossPlan cross_fwd_plan(int dtype, const CrossShape &c);
size_t cross_fwd_bytes(const CrossShape &c, const CrossPlan &p);
hipError_t cross_fwd(int dtype, const CrossArgs &a, const CrossShape &c, const CrossPlan &p, void *ws, hipStream_t st);
CrossBwdPlan cross_bwd_plan(int dtype, const CrossShape &c, bool dkv);
size_t cross_bwd_bytes(const CrossShape &c, const CrossBwdPlan &p);
hipError_t cross_bwd(int dtype, const CrossArgs &a, const CrossShape &c, const CrossBwdPlan &p, void *ws, hipStream_t st);
// bf16 on the matrix cores; fp32 on the fp32 matrix instruction
hipError_t cross_mfma_fwd(const CrossArgs &a, const CrossPlan &p, hipStream_t st);
hipError_t cross_mfma_bwd(const CrossArgs &a, const CrossBwdPlan &p, hipStream_t st);
hipError_t cross_f32_fwd(const CrossArgs &a, const CrossPlan &p, hipStream_t st);
hipError_t cross_f32_bwd(const CrossArgs &a, const CrossBwdPlan &p, hipStream_t st);

}  // namespace mmt
