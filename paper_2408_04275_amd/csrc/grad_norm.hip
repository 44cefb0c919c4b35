// Global gradient norm over many tensors, and clipping.
#include "ops.h"

namespace mmt {
namespace {

// the tensor that holds chunk k
__device__ __forceinline__ int tensor_of(const GradBatch &b, int k) {
    int lo = 0, hi = b.count;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (b.first[mid] <= k) lo = mid; else hi = mid;
    }
    return lo;
}

__device__ __forceinline__ double block_sum_f64(double v, double *red) {
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o, 64);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
    __syncthreads();
    return ((red[0] + red[1]) + (red[2] + red[3]));
}

__global__ __launch_bounds__(256) void grad_sum_sq_kernel(GradBatch b, double *part) {
    __shared__ double red[4];
    double q = 0.0;
    for (int k = blockIdx.x; k < b.first[b.count]; k += gridDim.x) {
        const int i = tensor_of(b, k);
        const long c0 = (long)(k - b.first[i]) * GRAD_CHUNK, c1 = min(c0 + GRAD_CHUNK, b.n[i]);
        for (long e = c0 + threadIdx.x; e < c1; e += 256) {
            const double g = b.in_f32[i] ? ((const float *)b.in[i])[e] : bf16_to_f32(((const bf16_t *)b.in[i])[e]);
            q += g * g;
        }
    }
    q = block_sum_f64(q, red);
    if (threadIdx.x == 0) part[blockIdx.x] = q;
}

__global__ __launch_bounds__(256) void grad_norm_finish_kernel(const double *part, int n, float max_norm, bool add, GradResult *result) {
    __shared__ double red[4];
    double q = 0.0;
    for (int i = threadIdx.x; i < n; i += 256) q += part[i];
    q = block_sum_f64(q, red);
    if (threadIdx.x != 0) return;
    if (add) q += result->sum_sq;
    const double norm = sqrt(q);
    result->sum_sq = q;
    result->norm = (float)norm;
    result->factor = !(norm < INFINITY) ? NAN : norm > (double)max_norm ? (float)((double)max_norm / norm) : 1.f;
}

__global__ __launch_bounds__(256) void grad_clip_kernel(GradBatch b, const GradResult *result) {
    float f = result->factor;
    const bool keep = f != f || f == 1.f;
    if (keep) f = 1.f;
    for (int k = blockIdx.x; k < b.first[b.count]; k += gridDim.x) {
        const int i = tensor_of(b, k);
        if (keep && b.in[i] == b.out[i]) continue;
        const long c0 = (long)(k - b.first[i]) * GRAD_CHUNK, c1 = min(c0 + GRAD_CHUNK, b.n[i]);
        for (long e = c0 + threadIdx.x; e < c1; e += 256) {
            const float g = f * (b.in_f32[i] ? ((const float *)b.in[i])[e] : bf16_to_f32(((const bf16_t *)b.in[i])[e]));
            if (b.out_f32[i]) ((float *)b.out[i])[e] = g;
            else ((bf16_t *)b.out[i])[e] = f32_to_bf16(g);
        }
    }
}

}  // namespace

int grad_norm_blocks(const GradBatch &b) { return b.first[b.count] < GRAD_BLOCKS ? b.first[b.count] : GRAD_BLOCKS; }

hipError_t grad_sum_sq(const GradBatch &b, double *part, hipStream_t st) {
    grad_sum_sq_kernel<<<grad_norm_blocks(b), 256, 0, st>>>(b, part);
    return hipGetLastError();
}

hipError_t grad_norm_finish(const double *part, int n, float max_norm, bool add, GradResult *result, hipStream_t st) {
    grad_norm_finish_kernel<<<1, 256, 0, st>>>(part, n, max_norm, add, result);
    return hipGetLastError();
}

hipError_t grad_clip(const GradBatch &b, const GradResult *result, hipStream_t st) {
    const int all = b.first[b.count];
    grad_clip_kernel<<<all < 2048 ? all : 2048, 256, 0, st>>>(b, result);
    return hipGetLastError();
}

}  // namespace mmt
