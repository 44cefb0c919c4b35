// C-ABI of the operators in mmtrain_ops.h: argument validation (host only, before any HIP call) and launches.
#include "../../include/mmtrain_ops.h"
#include "ops.h"
#include "api_checks.h"
#include <algorithm>
#include <cmath>

using namespace mmt;

namespace {

bool is_dtype(int32_t d) { return d == MMTRAIN_F32 || d == MMTRAIN_BF16; }

// ---- rotary positions ----------------------------------------------------------------
int rope_turns(const mmtrain_rope_desc &d, RopeArgs &a) {
    const double two_pi = 6.283185307179586476925;
    const bool blended = d.scaling == MMTRAIN_ROPE_WAVELENGTH || d.scaling == MMTRAIN_ROPE_RAMP;
    if (d.scaling != MMTRAIN_ROPE_PLAIN && !(d.factor >= 1.f && std::isfinite(d.factor))) return MMTRAIN_ERR_INVALID_ARG;
    if (blended && !(d.low > 0.f && d.high > d.low && std::isfinite(d.high) && d.orig_context > 0.f && std::isfinite(d.orig_context))) return MMTRAIN_ERR_INVALID_ARG;
    const double base = d.base, r = d.rot_dim, s = d.factor, context = d.orig_context;
    double first = 0.0, last = 0.0;
    if (d.scaling == MMTRAIN_ROPE_RAMP) {
        auto index = [&](double turns) { return r * std::log(context / (two_pi * turns)) / (2.0 * std::log(base)); };
        first = std::max(std::floor(index(d.high)), 0.0);
        last = std::min(std::ceil(index(d.low)), r - 1.0);
    }
    // base^(-2 i / r) as exp(rate i): 2^-53 |ln theta| off instead of the 2^-53 of a power, bits that fp32 does not have (64 pairs on the host 1.4 -> 0.6 us)
    const double rate = -2.0 * std::log(base) / r;
    for (int i = 0; i < a.half; ++i) {
        double theta = std::exp(rate * i), keep = 1.0;
        if (d.scaling == MMTRAIN_ROPE_LINEAR) keep = 0.0;
        else if (d.scaling == MMTRAIN_ROPE_WAVELENGTH) keep = (context * theta / two_pi - d.low) / ((double)d.high - d.low);
        else if (d.scaling == MMTRAIN_ROPE_RAMP) keep = 1.0 - (i - first) / std::max(last - first, 1e-3);
        keep = std::min(std::max(keep, 0.0), 1.0);
        if (keep < 1.0) theta *= keep + (1.0 - keep) / s;
        a.turns[i] = theta / two_pi;
    }
    return MMTRAIN_OK;
}

// ---- the join of branch and residual stream ----------------------------------------------
int check_join(const mmtrain_residual_norm_desc *d) {
    if (!d || d->struct_size != sizeof(mmtrain_residual_norm_desc) || !is_dtype(d->dtype)) return MMTRAIN_ERR_INVALID_ARG;
    for (int k : {d->post_norm, d->pre_norm})
        if (k < MMTRAIN_NORM_NONE || k > MMTRAIN_NORM_LAYER) return MMTRAIN_ERR_INVALID_ARG;
    if (d->gate < MMTRAIN_GATE_NONE || d->gate > MMTRAIN_GATE_SEGMENT || d->hidden <= 0) return MMTRAIN_ERR_INVALID_ARG;
    if (d->post_norm != MMTRAIN_NORM_NONE && !(d->post_eps > 0.f)) return MMTRAIN_ERR_INVALID_ARG;
    if (d->pre_norm != MMTRAIN_NORM_NONE && !(d->pre_eps > 0.f)) return MMTRAIN_ERR_INVALID_ARG;
    if (!std::isfinite(d->residual_scale) || !std::isfinite(d->branch_scale)) return MMTRAIN_ERR_INVALID_ARG;
    if (d->hidden % 8 || d->hidden > 8192) return MMTRAIN_ERR_UNSUPPORTED;
    return MMTRAIN_OK;
}

// What forward and backward have in common: the description, the segments of a segment gate, and that parameters are there
// exactly where the description has them
int join_common(const mmtrain_residual_norm_desc *d, int32_t T, const mmtrain_batch *batch, const mmtrain_residual_norm_weights *w, JoinArgs &a) {
    int rc = check_join(d);
    if (rc) return rc;
    if (T < 0 || !w) return MMTRAIN_ERR_INVALID_ARG;
    if (T > JOIN_MAX_ROWS) return MMTRAIN_ERR_UNSUPPORTED;
    a = JoinArgs{};
    a.T = T; a.H = d->hidden; a.post = d->post_norm; a.pre = d->pre_norm; a.gate = d->gate;
    a.post_eps = d->post_eps; a.pre_eps = d->pre_eps; a.alpha = d->residual_scale; a.beta = d->branch_scale;
    if (d->gate == MMTRAIN_GATE_SEGMENT) {
        if ((rc = check_batch(batch))) return rc;
        if (batch->total_tokens != T) return MMTRAIN_ERR_BAD_SEGMENTS;
        if (batch->n_segments > JOIN_MAX_SEGMENTS) return MMTRAIN_ERR_UNSUPPORTED;
        a.cu = batch->cu_seqlens_dev; a.S = batch->n_segments;
        if (a.S > 0 && !a.cu) return MMTRAIN_ERR_INVALID_ARG;
    }
    if (!w->post_w != (d->post_norm == MMTRAIN_NORM_NONE) || !w->post_b != (d->post_norm != MMTRAIN_NORM_LAYER) ||
        !w->pre_w != (d->pre_norm == MMTRAIN_NORM_NONE) || !w->pre_b != (d->pre_norm != MMTRAIN_NORM_LAYER) ||
        !w->gate != (d->gate == MMTRAIN_GATE_NONE))
        return MMTRAIN_ERR_INVALID_ARG;
    if (misaligned({w->post_w, w->post_b, w->gate, w->pre_w, w->pre_b})) return MMTRAIN_ERR_INVALID_ARG;
    a.post_w = w->post_w; a.post_b = w->post_b; a.gate_v = w->gate; a.pre_w = w->pre_w; a.pre_b = w->pre_b;
    return MMTRAIN_OK;
}

// Partial sums of the parameters' gradients, one array after the other
size_t join_parts(const mmtrain_residual_norm_desc &d, int32_t T, uint8_t *base, JoinArgs &a) {
    const size_t rows = (size_t)join_bwd_blocks(T, d.hidden) * d.hidden;
    size_t off = 0;
    auto take = [&](bool used, size_t n) -> float * {
        if (!used) return nullptr;
        float *p = base ? reinterpret_cast<float *>(base + off) : nullptr;
        off += (n * sizeof(float) + 255) & ~size_t(255);
        return p;
    };
    a.p_post_w = take(d.post_norm != MMTRAIN_NORM_NONE, rows);
    a.p_post_b = take(d.post_norm == MMTRAIN_NORM_LAYER, rows);
    a.p_pre_w = take(d.pre_norm != MMTRAIN_NORM_NONE, rows);
    a.p_pre_b = take(d.pre_norm == MMTRAIN_NORM_LAYER, rows);
    a.p_gate = take(d.gate != MMTRAIN_GATE_NONE, d.gate == MMTRAIN_GATE_SEGMENT ? 2 * rows : rows);
    return off + 256;
}

// ---- gradient norm and clipping -----------------------------------------------------------
constexpr int64_t GRAD_MAX_ELEMENTS = (int64_t)1 << 36;          // a tensor: chunks of a batch are counted in 32 bits

int check_tensors(const mmtrain_grad_tensor *t, int32_t n, bool clip) {
    if (n < 0 || (n > 0 && !t)) return MMTRAIN_ERR_INVALID_ARG;
    for (int32_t i = 0; i < n; ++i) {
        if (t[i].n < 0 || !is_dtype(t[i].dtype)) return MMTRAIN_ERR_INVALID_ARG;
        if (t[i].n > GRAD_MAX_ELEMENTS) return MMTRAIN_ERR_UNSUPPORTED;
        if (t[i].n > 0 && !t[i].grad) return MMTRAIN_ERR_INVALID_ARG;
        if (misaligned({t[i].grad})) return MMTRAIN_ERR_INVALID_ARG;
        if (!clip || !t[i].out) continue;
        if (!is_dtype(t[i].out_dtype) || misaligned({t[i].out})) return MMTRAIN_ERR_INVALID_ARG;
        if (t[i].out == t[i].grad && t[i].out_dtype != t[i].dtype) return MMTRAIN_ERR_INVALID_ARG;
    }
    return MMTRAIN_OK;
}

// ---- whether what one tensor writes is memory of another one, or of its own gradient in another place than in place ----
struct Range { uintptr_t a, b; bool written; };

// A tensor's gradient, and behind it what is written in another place
int ranges_of(const mmtrain_grad_tensor &t, Range *r) {
    if (t.n == 0) return 0;
    auto end = [&](uintptr_t p, int32_t dtype) { return p + (uintptr_t)t.n * (dtype == MMTRAIN_F32 ? 4 : 2); };
    const uintptr_t g = (uintptr_t)t.grad, o = (uintptr_t)t.out;
    const bool in_place = !o || o == g;
    r[0] = {g, end(g, t.dtype), in_place};
    if (in_place) return 1;
    r[1] = {o, end(o, t.out_dtype), true};
    return 2;
}

// Ranges in the order of their beginnings: whether one meets a range before it, one of the two written
struct Sweep {
    uintptr_t end = 0, end_written = 0;                     // of the ranges so far
    bool meets(const Range &x) {
        const bool hit = x.a < (x.written ? end : end_written);
        end = std::max(end, x.b);
        if (x.written) end_written = std::max(end_written, x.b);
        return hit;
    }
};

// Nothing is allocated.  Lists whose gradients stand in address order, and whose outputs do (parts of flat buffers), are merged as they are.  Others are
// sorted on the stack: in one piece where their ranges fit, else two parts of half as many at a time, every part beside every other.  us on the host, in order /
// shuffled: 288 tensors 3.4 / 10.8 (a list of the ranges on the heap: 10.6 / 13.4), 2000 25 / 258 (94 / 288), 10000 194 / 4160 (1166 / 1507).
constexpr int OVERLAP_RANGES = 8192;        // 128 KB

bool in_address_order(const mmtrain_grad_tensor *t, int32_t n) {
    uintptr_t last[2] = {0, 0};
    for (int32_t i = 0; i < n; ++i) {
        Range r[2];
        for (int k = 0, m = ranges_of(t[i], r); k < m; ++k) {
            if (r[k].a < last[k]) return false;
            last[k] = r[k].a;
        }
    }
    return true;
}

bool ordered_overlap(const mmtrain_grad_tensor *t, int32_t n) {
    Sweep sweep;
    int32_t i = 0, j = 0;                                   // next gradient, next output in another place
    for (;;) {
        Range g[2], o[2];
        while (i < n && ranges_of(t[i], g) == 0) ++i;
        while (j < n && ranges_of(t[j], o) < 2) ++j;
        if (i >= n && j >= n) return false;
        const bool gradient = j >= n || (i < n && g[0].a <= o[1].a);
        if (sweep.meets(gradient ? g[0] : o[1])) return true;
        ++(gradient ? i : j);
    }
}

// The ranges of tensors [first, last) in the order of their beginnings: 2 (tensor - first), and 1 more for an output
struct Begin { uintptr_t a; uint32_t which; };

int sorted_ranges(const mmtrain_grad_tensor *t, int64_t first, int64_t last, Begin *order) {
    int count = 0;
    for (int64_t i = first; i < last; ++i) {
        Range r[2];
        for (int k = 0, m = ranges_of(t[i], r); k < m; ++k) order[count++] = {r[k].a, (uint32_t)(2 * (i - first) + k)};
    }
    std::sort(order, order + count, [](const Begin &x, const Begin &y) { return x.a < y.a; });
    return count;
}

Range range(const mmtrain_grad_tensor *t, int64_t first, const Begin &x) {
    Range r[2];
    ranges_of(t[first + x.which / 2], r);
    return r[x.which & 1];
}

bool outputs_overlap(const mmtrain_grad_tensor *t, int32_t n) {
    if (in_address_order(t, n)) return ordered_overlap(t, n);
    Begin order[OVERLAP_RANGES];
    if (n <= OVERLAP_RANGES / 2) {
        const int count = sorted_ranges(t, 0, n, order);
        Sweep sweep;
        for (int i = 0; i < count; ++i)
            if (sweep.meets(range(t, 0, order[i]))) return true;
        return false;
    }
    constexpr int PART = OVERLAP_RANGES / 4;                // tensors
    Begin *other = order + OVERLAP_RANGES / 2;
    for (int64_t p = 0; p + PART < n; p += PART) {
        const int mine = sorted_ranges(t, p, p + PART, order);
        for (int64_t q = p + PART; q < n; q += PART) {      // (a part's own ranges meet beside any other part)
            const int theirs = sorted_ranges(t, q, std::min<int64_t>(q + PART, n), other);
            Sweep sweep;
            for (int i = 0, j = 0; i < mine || j < theirs;) {
                const bool first = j >= theirs || (i < mine && order[i].a <= other[j].a);
                if (sweep.meets(first ? range(t, p, order[i]) : range(t, q, other[j]))) return true;
                ++(first ? i : j);
            }
        }
    }
    return false;
}

// The tensors in batches of N, each handed to launch(); empty tensors are left out
template <int N, typename F>
int for_batches_of(const mmtrain_grad_tensor *t, int32_t n, F launch) {
    GradBatch<N> b;
    b.count = 0;
    for (int32_t k = 0; k < n; ++k) {
        const mmtrain_grad_tensor &g = t[k];
        if (g.n == 0) continue;
        const int i = b.count++;
        b.in[i] = g.grad; b.out[i] = g.out ? g.out : const_cast<void *>(g.grad);
        b.n[i] = g.n;
        b.in_f32[i] = g.dtype == MMTRAIN_F32;
        b.out_f32[i] = (g.out ? g.out_dtype : g.dtype) == MMTRAIN_F32;
        if (b.count < N) continue;
        grad_chunks(b);
        HIP_TRY(launch(b));
        b.count = 0;
    }
    if (b.count) {
        grad_chunks(b);
        HIP_TRY(launch(b));
    }
    return MMTRAIN_OK;
}

template <typename F>
int for_batches(const mmtrain_grad_tensor *t, int32_t n, F launch) {
    return n <= GRAD_FEW ? for_batches_of<GRAD_FEW>(t, n, launch) : for_batches_of<GRAD_BATCH>(t, n, launch);
}

}  // namespace

extern "C" {

int mmtrain_rope(const mmtrain_rope_desc *desc, int32_t n_tokens, const mmtrain_batch *batch, const int32_t *positions_dev,
                 const void *x, int64_t ld_x, void *y, int64_t ld_y, uint32_t flags, void *hip_stream) {
    if (!desc || desc->struct_size != sizeof(mmtrain_rope_desc) || !is_dtype(desc->dtype)) return MMTRAIN_ERR_INVALID_ARG;
    if (desc->layout != MMTRAIN_ROPE_HALF && desc->layout != MMTRAIN_ROPE_INTERLEAVED) return MMTRAIN_ERR_INVALID_ARG;
    if (desc->scaling < MMTRAIN_ROPE_PLAIN || desc->scaling > MMTRAIN_ROPE_RAMP) return MMTRAIN_ERR_INVALID_ARG;
    if (desc->n_heads <= 0 || desc->head_dim <= 0 || desc->rot_dim <= 0 || desc->rot_dim > desc->head_dim) return MMTRAIN_ERR_INVALID_ARG;
    if (!(desc->base > 1.f && std::isfinite(desc->base)) || !(desc->magnitude >= 0.f && std::isfinite(desc->magnitude))) return MMTRAIN_ERR_INVALID_ARG;
    if (desc->rot_dim % 2 || desc->head_dim > 2 * ROPE_MAX_HALF || desc->n_heads > ROPE_MAX_HEADS) return MMTRAIN_ERR_UNSUPPORTED;
    RopeArgs a = {};
    a.half = desc->rot_dim / 2;
    int rc = rope_turns(*desc, a);
    if (rc) return rc;
    if (n_tokens < 0 || (flags & ~MMTRAIN_ROPE_GRADIENT) || (batch && positions_dev)) return MMTRAIN_ERR_INVALID_ARG;
    if (batch) {
        if ((rc = check_batch(batch))) return rc;
        if (batch->total_tokens != n_tokens) return MMTRAIN_ERR_BAD_SEGMENTS;
        a.cu = batch->cu_seqlens_dev; a.S = batch->n_segments;
    }
    const int64_t row = (int64_t)desc->n_heads * desc->head_dim;
    if (ld_x < row || ld_y < row) return MMTRAIN_ERR_INVALID_ARG;
    if (n_tokens == 0) return MMTRAIN_OK;
    if ((!batch && !positions_dev) || !x || !y || misaligned({x, y}) || ((uintptr_t)positions_dev & 3)) return MMTRAIN_ERR_INVALID_ARG;
    if (x == y && ld_x != ld_y) return MMTRAIN_ERR_INVALID_ARG;
    a.T = n_tokens; a.heads = desc->n_heads; a.d = desc->head_dim;
    a.interleaved = desc->layout == MMTRAIN_ROPE_INTERLEAVED;
    a.positions = positions_dev; a.x = x; a.ldx = ld_x; a.y = y; a.ldy = ld_y;
    double m = desc->magnitude;
    if (m == 0.0) m = desc->scaling == MMTRAIN_ROPE_RAMP ? 0.1 * std::log((double)desc->factor) + 1.0 : 1.0;
    a.cos_scale = (float)m;
    a.sin_scale = (flags & MMTRAIN_ROPE_GRADIENT) ? -(float)m : (float)m;
    HIP_TRY(rope(desc->dtype, a, (hipStream_t)hip_stream));
    return MMTRAIN_OK;
}

size_t mmtrain_residual_norm_workspace_bytes(const mmtrain_residual_norm_desc *desc, int32_t n_tokens) {
    if (check_join(desc) != MMTRAIN_OK || n_tokens < 0) return 0;
    JoinArgs a = {};
    return join_parts(*desc, n_tokens, nullptr, a);
}

int mmtrain_residual_norm_fwd(const mmtrain_residual_norm_desc *desc, int32_t n_tokens, const mmtrain_batch *batch,
                              const mmtrain_residual_norm_weights *weights, const void *x, const void *branch, void *y, void *h,
                              const mmtrain_residual_norm_stats *stats, void *hip_stream) {
    JoinArgs a;
    int rc = join_common(desc, n_tokens, batch, weights, a);
    if (rc || n_tokens == 0) return rc;
    if (!x || !branch != !y || !h != (desc->pre_norm == MMTRAIN_NORM_NONE)) return MMTRAIN_ERR_INVALID_ARG;
    if (!branch && (desc->post_norm != MMTRAIN_NORM_NONE || desc->gate != MMTRAIN_GATE_NONE || !h)) return MMTRAIN_ERR_INVALID_ARG;
    if (branch == x || (branch && y == branch) || (h && (h == x || h == branch || h == y))) return MMTRAIN_ERR_INVALID_ARG;
    if (misaligned({x, branch, y, h})) return MMTRAIN_ERR_INVALID_ARG;
    if (stats) {
        if (misaligned({stats->post_mean, stats->post_rstd, stats->pre_mean, stats->pre_rstd})) return MMTRAIN_ERR_INVALID_ARG;
        a.post_mean = stats->post_mean; a.post_rstd = stats->post_rstd; a.pre_mean = stats->pre_mean; a.pre_rstd = stats->pre_rstd;
    }
    a.x = x; a.b = branch; a.y = y; a.h = h;
    HIP_TRY(join_fwd(desc->dtype, a, (hipStream_t)hip_stream));
    return MMTRAIN_OK;
}

int mmtrain_residual_norm_bwd(const mmtrain_residual_norm_desc *desc, int32_t n_tokens, const mmtrain_batch *batch,
                              const mmtrain_residual_norm_weights *weights, const void *y, const void *branch,
                              const mmtrain_residual_norm_stats *stats, const void *dy, const void *dh, void *dx, void *d_branch,
                              const mmtrain_residual_norm_grads *grads, uint32_t flags, void *workspace, size_t workspace_bytes,
                              void *hip_stream) {
    JoinArgs a;
    int rc = join_common(desc, n_tokens, batch, weights, a);
    if (rc) return rc;
    if (flags & ~(MMTRAIN_BWD_ACCUMULATE_WGRAD | MMTRAIN_BWD_WGRAD_F32)) return MMTRAIN_ERR_INVALID_ARG;
    const bool pre = desc->pre_norm != MMTRAIN_NORM_NONE, post = desc->post_norm != MMTRAIN_NORM_NONE, gate = desc->gate != MMTRAIN_GATE_NONE;
    const mmtrain_residual_norm_grads none = {};
    const mmtrain_residual_norm_grads &g = grads ? *grads : none;
    if ((g.post_w && !post) || (g.post_b && desc->post_norm != MMTRAIN_NORM_LAYER) || (g.pre_w && !pre) ||
        (g.pre_b && desc->pre_norm != MMTRAIN_NORM_LAYER) || (g.gate && !gate))
        return MMTRAIN_ERR_INVALID_ARG;
    if (misaligned({g.post_w, g.post_b, g.gate, g.pre_w, g.pre_b})) return MMTRAIN_ERR_INVALID_ARG;
    const bool any = g.post_w || g.post_b || g.gate || g.pre_w || g.pre_b;
    if (n_tokens > 0) {
        if (!dh != !pre || (!dh && !dy) || (pre && !y) || (!branch && (post || gate || d_branch || !pre))) return MMTRAIN_ERR_INVALID_ARG;
        if (misaligned({y, branch, dy, dh, dx, d_branch})) return MMTRAIN_ERR_INVALID_ARG;
        if (dx && (dx == y || dx == branch || dx == dh || dx == d_branch)) return MMTRAIN_ERR_INVALID_ARG;
        if (d_branch && (d_branch == y || d_branch == branch || d_branch == dy)) return MMTRAIN_ERR_INVALID_ARG;
        if (pre || post) {
            if (!stats) return MMTRAIN_ERR_INVALID_ARG;
            if ((pre && !stats->pre_rstd) || (post && !stats->post_rstd) || (desc->pre_norm == MMTRAIN_NORM_LAYER && !stats->pre_mean) ||
                (desc->post_norm == MMTRAIN_NORM_LAYER && !stats->post_mean))
                return MMTRAIN_ERR_INVALID_ARG;
            if (misaligned({stats->post_mean, stats->post_rstd, stats->pre_mean, stats->pre_rstd})) return MMTRAIN_ERR_INVALID_ARG;
            a.post_mean = stats->post_mean; a.post_rstd = stats->post_rstd; a.pre_mean = stats->pre_mean; a.pre_rstd = stats->pre_rstd;
        }
    }
    if ((uintptr_t)workspace & 255) return MMTRAIN_ERR_INVALID_ARG;
    if (any && (!workspace || workspace_bytes < mmtrain_residual_norm_workspace_bytes(desc, n_tokens))) return MMTRAIN_ERR_WORKSPACE;
    if (any) join_parts(*desc, n_tokens, (uint8_t *)workspace, a);
    if (!g.post_w) a.p_post_w = nullptr;
    if (!g.post_b) a.p_post_b = nullptr;
    if (!g.pre_w) a.p_pre_w = nullptr;
    if (!g.pre_b) a.p_pre_b = nullptr;
    if (!g.gate) a.p_gate = nullptr;
    a.y = const_cast<void *>(y); a.b = branch; a.dy = dy; a.dh = dh; a.dx = dx; a.db = d_branch;
    a.grad_f32 = desc->dtype == MMTRAIN_F32 || (flags & MMTRAIN_BWD_WGRAD_F32);
    a.accumulate = (flags & MMTRAIN_BWD_ACCUMULATE_WGRAD) != 0;
    a.d_post_w = g.post_w; a.d_post_b = g.post_b; a.d_gate = g.gate; a.d_pre_w = g.pre_w; a.d_pre_b = g.pre_b;
    HIP_TRY(join_bwd(desc->dtype, a, (hipStream_t)hip_stream));
    return MMTRAIN_OK;
}

size_t mmtrain_grad_norm_workspace_bytes(int32_t n_tensors) {
    if (n_tensors < 0) return 0;
    return ((size_t)n_tensors / GRAD_BATCH + 1) * GRAD_BLOCKS * sizeof(double);
}

int mmtrain_grad_norm(const mmtrain_grad_tensor *tensors, int32_t n_tensors, float max_norm, uint32_t flags,
                      mmtrain_grad_norm_result *result, void *workspace, size_t workspace_bytes, void *hip_stream) {
    int rc = check_tensors(tensors, n_tensors, false);
    if (rc) return rc;
    if (!(max_norm >= 0.f) || (flags & ~MMTRAIN_GRAD_NORM_ADD) || !result || misaligned({result}) || ((uintptr_t)workspace & 255))
        return MMTRAIN_ERR_INVALID_ARG;
    if (!workspace || workspace_bytes < mmtrain_grad_norm_workspace_bytes(n_tensors)) return MMTRAIN_ERR_WORKSPACE;
    hipStream_t st = (hipStream_t)hip_stream;
    double *part = (double *)workspace;
    int parts = 0;
    rc = for_batches(tensors, n_tensors, [&](const auto &b) {
        const hipError_t e = grad_sum_sq(b, part + parts, st);
        parts += grad_norm_blocks(b);
        return e;
    });
    if (rc) return rc;
    HIP_TRY(grad_norm_finish(part, parts, max_norm, (flags & MMTRAIN_GRAD_NORM_ADD) != 0, reinterpret_cast<GradResult *>(result), st));
    return MMTRAIN_OK;
}

int mmtrain_grad_clip(const mmtrain_grad_tensor *tensors, int32_t n_tensors, const mmtrain_grad_norm_result *result, void *hip_stream) {
    int rc = check_tensors(tensors, n_tensors, true);
    if (rc) return rc;
    if (!result || misaligned({result})) return MMTRAIN_ERR_INVALID_ARG;
    if (outputs_overlap(tensors, n_tensors)) return MMTRAIN_ERR_INVALID_ARG;
    size_t written = 0;
    for (int32_t i = 0; i < n_tensors; ++i) written += (size_t)tensors[i].n * ((tensors[i].out ? tensors[i].out_dtype : tensors[i].dtype) == MMTRAIN_F32 ? 4 : 2);
    return for_batches(tensors, n_tensors, [&](const auto &b) {
        return grad_clip(b, reinterpret_cast<const GradResult *>(result), grad_clip_streams(written), (hipStream_t)hip_stream);
    });
}

}  // extern "C"
