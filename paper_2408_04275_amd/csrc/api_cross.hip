// C-ABI of cross attention: argument validation (host only, before any HIP call) and launches.
#include "../../include/mmtrain_ops.h"
#include "ops.h"
#include "api_checks.h"
#include <cmath>

using namespace mmt;

namespace {

constexpr int64_t MAX_STRIDE = (int64_t)1 << 24;                // 64 rows stay within 32-bit byte offsets

int check_cross(const mmtrain_cross_attn_desc *d) {
    if (!d || d->struct_size != sizeof(mmtrain_cross_attn_desc) || (d->dtype != MMTRAIN_F32 && d->dtype != MMTRAIN_BF16)) return MMTRAIN_ERR_INVALID_ARG;
    if (d->n_heads <= 0 || d->n_kv_heads <= 0 || d->head_dim <= 0 || !(d->softmax_scale >= 0.f && std::isfinite(d->softmax_scale))) return MMTRAIN_ERR_INVALID_ARG;
    if (d->head_dim % 16 || d->head_dim > 128 || d->n_heads % d->n_kv_heads || d->n_heads > 4096) return MMTRAIN_ERR_UNSUPPORTED;
    return MMTRAIN_OK;
}

// ordered: kv_begin and kv_end have to be non-decreasing over the runs that see something
int check_cross_batch(const mmtrain_cross_batch *b, bool ordered) {
    if (!b || b->q_tokens < 0 || b->kv_tokens < 0 || b->n_segments < 0 || !b->cu_q_host) return MMTRAIN_ERR_INVALID_ARG;
    if (b->n_segments > 0 && (!b->kv_begin_host || !b->kv_end_host)) return MMTRAIN_ERR_INVALID_ARG;
    if (b->n_segments > CROSS_MAX_SEGMENTS || b->q_tokens > 1 << 28 || b->kv_tokens > 1 << 30) return MMTRAIN_ERR_UNSUPPORTED;
    const int32_t *cu = b->cu_q_host, *lo = b->kv_begin_host, *hi = b->kv_end_host;
    if (cu[0] != 0) return MMTRAIN_ERR_BAD_SEGMENTS;
    int32_t last_lo = 0, last_hi = 0;
    for (int s = 0; s < b->n_segments; ++s) {
        if (cu[s + 1] < cu[s] || lo[s] < 0 || hi[s] < lo[s] || hi[s] > b->kv_tokens) return MMTRAIN_ERR_BAD_SEGMENTS;
        if (!ordered || lo[s] == hi[s]) continue;
        if (lo[s] < last_lo || hi[s] < last_hi) return MMTRAIN_ERR_BAD_SEGMENTS;
        last_lo = lo[s]; last_hi = hi[s];
    }
    if (cu[b->n_segments] != b->q_tokens) return MMTRAIN_ERR_BAD_SEGMENTS;
    if (b->n_segments > 0 && (!b->cu_q_dev || !b->kv_begin_dev || !b->kv_end_dev)) return MMTRAIN_ERR_INVALID_ARG;
    return MMTRAIN_OK;
}

// rows of a run and key/value head, log-sum-exps of a group: 32-bit numbers and byte offsets; workgroups of up to 512 threads: fewer than 2^32 threads
int check_sizes(const mmtrain_cross_attn_desc &d, const mmtrain_cross_batch &b) {
    const int64_t S = b.n_segments, most = ((int64_t)1 << 23) - 2;
    const int rows = d.dtype == MMTRAIN_F32 ? 16 : 32, keys = d.dtype == MMTRAIN_F32 ? 16 : 128;
    return (int64_t)b.q_tokens * (d.n_heads / d.n_kv_heads) > 1 << 28 || ((int64_t)b.q_tokens + S) * d.n_heads > INT32_MAX ||
           (int64_t)b.q_tokens * d.n_heads / rows + S * d.n_kv_heads > most || (b.kv_tokens / keys + 128 / keys * (2 * S + 1)) * d.n_kv_heads > most
               ? MMTRAIN_ERR_UNSUPPORTED : MMTRAIN_OK;
}

int check_rows(const mmtrain_cross_attn_desc &d, int heads, const void *p, int64_t ld) {
    if (!p || misaligned({p}) || ld < (int64_t)heads * d.head_dim) return MMTRAIN_ERR_INVALID_ARG;
    return ld % (d.dtype == MMTRAIN_F32 ? 4 : 8) || ld >= MAX_STRIDE ? MMTRAIN_ERR_UNSUPPORTED : MMTRAIN_OK;
}

void fill(const mmtrain_cross_attn_desc &d, const mmtrain_cross_batch &b, CrossArgs &a) {
    a = CrossArgs{};
    a.Tq = b.q_tokens; a.Tk = b.kv_tokens; a.S = b.n_segments;
    a.nh = d.n_heads; a.nkv = d.n_kv_heads; a.d = d.head_dim;
    a.scale = d.softmax_scale > 0.f ? d.softmax_scale : 1.f / std::sqrt((float)d.head_dim);
    a.cu = b.cu_q_dev; a.begin = b.kv_begin_dev; a.end = b.kv_end_dev;
}

CrossShape shape_of(const mmtrain_cross_attn_desc &d, const mmtrain_cross_batch &b) {
    return {b.q_tokens, b.kv_tokens, b.n_segments, d.n_heads, d.n_kv_heads, d.head_dim, b.cu_q_host, b.kv_begin_host, b.kv_end_host};
}

// q, k, v and o as the calls have them in common (k and v: only where there are keys)
int tensors_of(const mmtrain_cross_attn_desc &d, const mmtrain_cross_attn_tensors *t, CrossArgs &a) {
    if (!t) return MMTRAIN_ERR_INVALID_ARG;
    int rc;
    if (a.Tq > 0 && ((rc = check_rows(d, a.nh, t->q, t->ld_q)) || (rc = check_rows(d, a.nh, t->o, t->ld_o)))) return rc;
    if (a.Tk > 0 && ((rc = check_rows(d, a.nkv, t->k, t->ld_k)) || (rc = check_rows(d, a.nkv, t->v, t->ld_v)))) return rc;
    if (misaligned({t->lse})) return MMTRAIN_ERR_INVALID_ARG;
    a.q = t->q; a.ldq = t->ld_q; a.k = t->k; a.ldk = t->ld_k; a.v = t->v; a.ldv = t->ld_v; a.o = t->o; a.ldo = t->ld_o; a.lse = t->lse;
    return MMTRAIN_OK;
}

}  // namespace

extern "C" {

size_t mmtrain_cross_attn_workspace_bytes(const mmtrain_cross_attn_desc *desc, const mmtrain_cross_batch *batch, int is_bwd) {
    if (check_cross(desc) || check_cross_batch(batch, false) || check_sizes(*desc, *batch)) return 0;
    const CrossShape c = shape_of(*desc, *batch);
    return (is_bwd ? cross_bwd_bytes(c, cross_bwd_plan(desc->dtype, c, check_cross_batch(batch, true) == MMTRAIN_OK)) : cross_fwd_bytes(c, cross_fwd_plan(desc->dtype, c))) + 256;
}

int mmtrain_cross_attn_fwd(const mmtrain_cross_attn_desc *desc, const mmtrain_cross_batch *batch, const mmtrain_cross_attn_tensors *tensors,
                           void *workspace, size_t workspace_bytes, void *hip_stream) {
    int rc = check_cross(desc);
    if (rc || (rc = check_cross_batch(batch, false)) || (rc = check_sizes(*desc, *batch))) return rc;
    CrossArgs a;
    fill(*desc, *batch, a);
    if ((rc = tensors_of(*desc, tensors, a))) return rc;
    if (a.Tq == 0) return MMTRAIN_OK;
    if (a.o == a.q || a.o == a.k || a.o == a.v) return MMTRAIN_ERR_INVALID_ARG;
    if ((uintptr_t)workspace & 255) return MMTRAIN_ERR_INVALID_ARG;
    const CrossShape c = shape_of(*desc, *batch);
    const CrossPlan plan = cross_fwd_plan(desc->dtype, c);
    if (!workspace || workspace_bytes < cross_fwd_bytes(c, plan) + 256) return MMTRAIN_ERR_WORKSPACE;
    HIP_TRY(cross_fwd(desc->dtype, a, c, plan, workspace, (hipStream_t)hip_stream));
    return MMTRAIN_OK;
}

int mmtrain_cross_attn_bwd(const mmtrain_cross_attn_desc *desc, const mmtrain_cross_batch *batch, const mmtrain_cross_attn_tensors *tensors,
                           const mmtrain_cross_attn_grads *grads, void *workspace, size_t workspace_bytes, void *hip_stream) {
    int rc = check_cross(desc);
    if (rc) return rc;
    if (!grads || !grads->d_k != !grads->d_v) return MMTRAIN_ERR_INVALID_ARG;
    if ((rc = check_cross_batch(batch, grads->d_k != nullptr)) || (rc = check_sizes(*desc, *batch))) return rc;
    CrossArgs a;
    fill(*desc, *batch, a);
    if ((rc = tensors_of(*desc, tensors, a))) return rc;
    const mmtrain_cross_attn_grads &g = *grads;
    if (a.Tq > 0 && (!a.lse || (rc = check_rows(*desc, a.nh, g.d_o, g.ld_do)))) return rc ? rc : MMTRAIN_ERR_INVALID_ARG;
    if (g.d_q && (rc = check_rows(*desc, a.nh, g.d_q, g.ld_dq))) return rc;
    if (g.d_k && ((rc = check_rows(*desc, a.nkv, g.d_k, g.ld_dk)) || (rc = check_rows(*desc, a.nkv, g.d_v, g.ld_dv)))) return rc;
    const void *const in[5] = {a.q, a.k, a.v, a.o, g.d_o}, *const out[3] = {g.d_q, g.d_k, g.d_v};
    for (int i = 0; i < 3; ++i) {
        for (const void *p : in)
            if (out[i] && out[i] == p) return MMTRAIN_ERR_INVALID_ARG;
        if (out[i] && out[i] == out[(i + 1) % 3]) return MMTRAIN_ERR_INVALID_ARG;
    }
    if ((uintptr_t)workspace & 255) return MMTRAIN_ERR_INVALID_ARG;
    const CrossShape c = shape_of(*desc, *batch);
    const CrossBwdPlan plan = cross_bwd_plan(desc->dtype, c, g.d_k != nullptr);
    if (!workspace || workspace_bytes < cross_bwd_bytes(c, plan) + 256) return MMTRAIN_ERR_WORKSPACE;
    a.d_o = g.d_o; a.lddo = g.ld_do;
    a.dq = g.d_q; a.lddq = g.ld_dq; a.dk = g.d_k; a.lddk = g.ld_dk; a.dv = g.d_v; a.lddv = g.ld_dv;
    HIP_TRY(cross_bwd(desc->dtype, a, c, plan, workspace, (hipStream_t)hip_stream));
    return MMTRAIN_OK;
}

}  // extern "C"
