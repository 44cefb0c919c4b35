// Attention of runs of queries to ranges of keys: one wavefront per query and head (forward, dQ) or key and key/value head (dK, dV),
// the head's features over its lanes.
#include "ops.h"

namespace mmt {
namespace {

template <typename T>
__device__ __forceinline__ void load_row(const T *p, int d, float (&v)[2]) {
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int e = 0; e < 2; ++e) v[e] = lane + 64 * e < d ? Elem<T>::load(p + lane + 64 * e) : 0.f;
}
template <typename T>
__device__ __forceinline__ void store_row(T *p, int d, const float (&v)[2], float scale) {
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int e = 0; e < 2; ++e)
        if (lane + 64 * e < d) Elem<T>::store(p + lane + 64 * e, v[e] * scale);
}
__device__ __forceinline__ float dot(const float (&a)[2], const float (&b)[2]) { return wave_sum(a[0] * b[0] + a[1] * b[1]); }

template <typename T>
__global__ __launch_bounds__(256) void cross_fwd_kernel(CrossArgs a) {
    const long w = (long)blockIdx.x * 4 + (threadIdx.x >> 6);
    if (w >= (long)a.Tq * a.nh) return;
    const int h = (int)(w % a.nh), t = (int)(w / a.nh), g = h / (a.nh / a.nkv), s = find_segment(a.cu, a.S, t);
    float q[2], k[2], v[2], acc[2] = {0.f, 0.f}, m = -INFINITY, l = 0.f;
    load_row((const T *)a.q + t * a.ldq + (long)h * a.d, a.d, q);
    for (int j = a.begin[s]; j < a.end[s]; ++j) {
        load_row((const T *)a.k + j * a.ldk + (long)g * a.d, a.d, k);
        load_row((const T *)a.v + j * a.ldv + (long)g * a.d, a.d, v);
        const float x = dot(q, k) * a.scale, mn = fmaxf(m, x), corr = expf(m - mn), p = expf(x - mn);
        l = l * corr + p;
#pragma unroll
        for (int e = 0; e < 2; ++e) acc[e] = acc[e] * corr + p * v[e];
        m = mn;
    }
    store_row((T *)a.o + t * a.ldo + (long)h * a.d, a.d, acc, l > 0.f ? 1.f / l : 0.f);
    if (a.lse && (threadIdx.x & 63) == 0) a.lse[(long)h * a.Tq + t] = m + logf(l);
}

template <typename T>
__global__ __launch_bounds__(256) void cross_dq_kernel(CrossArgs a) {
    const long w = (long)blockIdx.x * 4 + (threadIdx.x >> 6);
    if (w >= (long)a.Tq * a.nh) return;
    const int h = (int)(w % a.nh), t = (int)(w / a.nh), g = h / (a.nh / a.nkv), s = find_segment(a.cu, a.S, t);
    float q[2], k[2], v[2], go[2], o[2], dq[2] = {0.f, 0.f};
    load_row((const T *)a.q + t * a.ldq + (long)h * a.d, a.d, q);
    load_row((const T *)a.d_o + t * a.lddo + (long)h * a.d, a.d, go);
    load_row((const T *)a.o + t * a.ldo + (long)h * a.d, a.d, o);
    const float D = dot(go, o), lse = a.lse[(long)h * a.Tq + t];
    if ((threadIdx.x & 63) == 0) a.D[(long)h * a.Tq + t] = D;
    if (!a.dq) return;
    for (int j = a.begin[s]; j < a.end[s]; ++j) {
        load_row((const T *)a.k + j * a.ldk + (long)g * a.d, a.d, k);
        load_row((const T *)a.v + j * a.ldv + (long)g * a.d, a.d, v);
        const float ds = expf(dot(q, k) * a.scale - lse) * (dot(go, v) - D);
#pragma unroll
        for (int e = 0; e < 2; ++e) dq[e] += ds * k[e];
    }
    store_row((T *)a.dq + t * a.lddq + (long)h * a.d, a.d, dq, a.scale);
}

template <typename T>
__global__ __launch_bounds__(256) void cross_dkv_kernel(CrossArgs a) {
    const long w = (long)blockIdx.x * 4 + (threadIdx.x >> 6);
    if (w >= (long)a.Tk * a.nkv) return;
    const int g = (int)(w % a.nkv), j = (int)(w / a.nkv), group = a.nh / a.nkv;
    float q[2], k[2], v[2], go[2], dk[2] = {0.f, 0.f}, dv[2] = {0.f, 0.f};
    load_row((const T *)a.k + j * a.ldk + (long)g * a.d, a.d, k);
    load_row((const T *)a.v + j * a.ldv + (long)g * a.d, a.d, v);
    for (int s = 0; s < a.S; ++s) {
        if (j < a.begin[s] || j >= a.end[s]) continue;
        for (int t = a.cu[s]; t < a.cu[s + 1]; ++t)
            for (int h = g * group; h < (g + 1) * group; ++h) {
                load_row((const T *)a.q + t * a.ldq + (long)h * a.d, a.d, q);
                load_row((const T *)a.d_o + t * a.lddo + (long)h * a.d, a.d, go);
                const float p = expf(dot(q, k) * a.scale - a.lse[(long)h * a.Tq + t]);
                const float ds = p * (dot(go, v) - a.D[(long)h * a.Tq + t]);
#pragma unroll
                for (int e = 0; e < 2; ++e) { dv[e] += p * go[e]; dk[e] += ds * q[e]; }
            }
    }
    store_row((T *)a.dk + j * a.lddk + (long)g * a.d, a.d, dk, a.scale);
    store_row((T *)a.dv + j * a.lddv + (long)g * a.d, a.d, dv, 1.f);
}

}  // namespace

hipError_t cross_fwd(int dtype, const CrossArgs &a, hipStream_t st) {
    if (a.Tq == 0) return hipSuccess;
    const int grid = ceil_div((long)a.Tq * a.nh, 4);
    if (dtype == DT_F32) cross_fwd_kernel<float><<<grid, 256, 0, st>>>(a);
    else cross_fwd_kernel<bf16_t><<<grid, 256, 0, st>>>(a);
    return hipGetLastError();
}

hipError_t cross_bwd(int dtype, const CrossArgs &a, hipStream_t st) {
    const int gq = ceil_div((long)a.Tq * a.nh, 4), gk = ceil_div((long)a.Tk * a.nkv, 4);
    if (!gq && (!a.dk || !gk)) return hipSuccess;
    if (gq) {
        if (dtype == DT_F32) cross_dq_kernel<float><<<gq, 256, 0, st>>>(a);
        else cross_dq_kernel<bf16_t><<<gq, 256, 0, st>>>(a);
    }
    if (a.dk && gk) {
        if (dtype == DT_F32) cross_dkv_kernel<float><<<gk, 256, 0, st>>>(a);
        else cross_dkv_kernel<bf16_t><<<gk, 256, 0, st>>>(a);
    }
    return hipGetLastError();
}

}  // namespace mmt
