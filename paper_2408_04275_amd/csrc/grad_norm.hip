// Global gradient norm over many tensors, and clipping.
//
// Memory-bound: the norm reads every gradient once, clipping reads and writes each once.  A launch takes up to GRAD_BATCH tensors, whose addresses
// it has as kernel arguments (nothing to copy, nothing to keep alive for a captured graph), cut into chunks that the workgroups take in turn; 64 bytes on
// their way per thread.
//
// Squares are added up in fp64: those of fp32 gradients leave the range of fp32 (a gradient of 1e20, or of 1e-23), and the conversions and fused
// multiply-adds, a quarter of what the vector ALUs can do while 5 TB/s arrive, cost nothing.  Every sum has a fixed order.
#include "ops.h"
#include <algorithm>

namespace mmt {
namespace {

// the tensor that holds chunk k
template <int N> __device__ __forceinline__ int tensor_of(const GradBatch<N> &b, int k) {
    int lo = 0, hi = b.count;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (b.first[mid] <= k) lo = mid; else hi = mid;
    }
    return lo;
}

template <int NT> __device__ __forceinline__ double block_sum_f64(double v, double *red) {
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o, 64);
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
    __syncthreads();
    double s = 0.0;
#pragma unroll
    for (int i = 0; i < NT / 64; ++i) s += red[i];
    return s;
}

// N neighbouring elements of a tensor
template <typename T, int N> struct Vec {
    uint32_t __attribute__((ext_vector_type(N * sizeof(T) / 4))) r;
    __device__ __forceinline__ float get(int i) const {
        if constexpr (sizeof(T) == 4) return __uint_as_float(r[i]);
        else return __uint_as_float(i & 1 ? r[i >> 1] & 0xffff0000u : r[i >> 1] << 16);
    }
};

// f(v, place) for the vectors of N elements of p[0 .. m), U requested together; tail(e) for the elements behind the last whole one
template <int N, int U, typename T, typename F, typename E>
__device__ __forceinline__ void for_vectors(const T *p, int m, F f, E tail) {
    typedef decltype(Vec<T, N>::r) raw;
    const raw *q = reinterpret_cast<const raw *>(p);
    const int nv = m / N;
    int v = threadIdx.x;
    for (; v + (U - 1) * 256 < nv; v += U * 256) {
        Vec<T, N> x[U];
#pragma unroll
        for (int u = 0; u < U; ++u) x[u].r = q[v + u * 256];
#pragma unroll
        for (int u = 0; u < U; ++u) f(x[u], v + u * 256);
    }
    for (; v < nv; v += 256) f(Vec<T, N>{q[v]}, v);
    if (nv * N + (int)threadIdx.x < m) tail(nv * N + threadIdx.x);
}

template <typename T> __device__ __forceinline__ void add_squares(const T *p, int m, double (&q)[2]) {
    constexpr int N = 16 / sizeof(T);
    for_vectors<N, 4>(p, m, [&](const Vec<T, N> &x, int) {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const double g = x.get(i);
            q[i & 1] += g * g;
        }
    }, [&](int e) {
        const double g = Elem<T>::load(p + e);
        q[0] += g * g;
    });
}

template <int N> __global__ __launch_bounds__(256) void grad_sum_sq_kernel(GradBatch<N> b, double *part) {
    __shared__ double red[4];
    double q[2] = {0.0, 0.0};
    for (int k = blockIdx.x; k < b.first[b.count]; k += gridDim.x) {
        const int i = tensor_of(b, k);
        const long at = (long)(k - b.first[i]) * b.chunk;
        const int m = (int)min((long)b.chunk, b.n[i] - at);
        if (b.in_f32[i]) add_squares((const float *)b.in[i] + at, m, q);
        else add_squares((const bf16_t *)b.in[i] + at, m, q);
    }
    const double s = block_sum_f64<256>(q[0] + q[1], red);
    if (threadIdx.x == 0) part[blockIdx.x] = s;
}

__global__ __launch_bounds__(1024) void grad_norm_finish_kernel(const double *part, int n, float max_norm, bool add, GradResult *result) {
    __shared__ double red[16];
    double q = 0.0;
    for (int i = threadIdx.x; i < n; i += 1024) q += part[i];
    q = block_sum_f64<1024>(q, red);
    if (threadIdx.x != 0) return;
    if (add) q += result->sum_sq;
    const double norm = sqrt(q);
    result->sum_sq = q;
    result->norm = (float)norm;
    result->factor = !((float)norm < INFINITY) ? NAN : norm > (double)max_norm ? (float)((double)max_norm / norm) : 1.f;
}

// A wavefront's stores cover whole lines: 16 bytes per lane of the wider type
template <bool STREAM, typename T, typename O> __device__ __forceinline__ void scale(const T *p, O *o, int m, float f) {
    constexpr int N = 16 / (sizeof(T) > sizeof(O) ? sizeof(T) : sizeof(O));
    for_vectors<N, 32 / (N * sizeof(T)) * 2>(p, m, [&](const Vec<T, N> &x, int v) {
        Vec<O, N> y;
#pragma unroll
        for (int i = 0; i < N; i += 4 / sizeof(O)) {
            if constexpr (sizeof(O) == 4) y.r[i] = __float_as_uint(f * x.get(i));
            else y.r[i / 2] = pack_bf16x2(f * x.get(i), f * x.get(i + 1));
        }
        decltype(y.r) *at = reinterpret_cast<decltype(y.r) *>(o) + v;
        if constexpr (STREAM) __builtin_nontemporal_store(y.r, at);
        else *at = y.r;
    }, [&](int e) { Elem<O>::store(o + e, f * Elem<T>::load(p + e)); });
}

template <bool STREAM, int N>
__global__ __launch_bounds__(256) void grad_clip_kernel(GradBatch<N> b, const GradResult *result) {
    float f = result->factor;
    const bool keep = f != f || f == 1.f;
    if (keep) f = 1.f;
    for (int k = blockIdx.x; k < b.first[b.count]; k += gridDim.x) {
        const int i = tensor_of(b, k);
        if (keep && b.in[i] == b.out[i]) continue;
        const long at = (long)(k - b.first[i]) * b.chunk;
        const int m = (int)min((long)b.chunk, b.n[i] - at);
        const float *p32 = (const float *)b.in[i] + at;
        const bf16_t *p16 = (const bf16_t *)b.in[i] + at;
        float *o32 = (float *)b.out[i] + at;
        bf16_t *o16 = (bf16_t *)b.out[i] + at;
        if (b.in_f32[i]) { if (b.out_f32[i]) scale<STREAM>(p32, o32, m, f); else scale<STREAM>(p32, o16, m, f); }
        else { if (b.out_f32[i]) scale<STREAM>(p16, o32, m, f); else scale<STREAM>(p16, o16, m, f); }
    }
}

}  // namespace

// Chunks of 2048 elements (one or two accesses a thread) as long as there are workgroups for them, up to 16384; longer ones only where their number
// would leave 32 bits
template <int N> void grad_chunks(GradBatch<N> &b) {
    long total = 0;
    for (int i = 0; i < b.count; ++i) total += b.n[i];
    long chunk = std::min(std::max((total / GRAD_BLOCKS + 2047) / 2048 * 2048, 2048l), 16384l);
    while (total / chunk > 0x3fffffff) chunk *= 2;
    b.chunk = (int)chunk;
    long first = 0;
    for (int i = 0; i < b.count; ++i) {
        b.first[i] = (int)first;
        first += (b.n[i] + chunk - 1) / chunk;
    }
    b.first[b.count] = (int)first;
}

template <int N> int grad_norm_blocks(const GradBatch<N> &b) { return std::min(b.first[b.count], GRAD_BLOCKS); }

template <int N> hipError_t grad_sum_sq(const GradBatch<N> &b, double *part, hipStream_t st) {
    grad_sum_sq_kernel<N><<<grad_norm_blocks(b), 256, 0, st>>>(b, part);
    return hipGetLastError();
}

hipError_t grad_norm_finish(const double *part, int n, float max_norm, bool add, GradResult *result, hipStream_t st) {
    grad_norm_finish_kernel<<<1, 1024, 0, st>>>(part, n, max_norm, add, result);
    return hipGetLastError();
}

// Streaming pays where what a call writes does not fit the memory-side cache (256 MB), where it would push out what is still to be read, and costs where
// the optimizer step that comes next finds it there.  us, plain -> streaming: norm and copy of 300 fp32 tensors (316 MB), alone 214 -> 177; copy from bf16
// to fp32 and optimizer step, 67 MB written 111 -> 120, 134 MB 200 -> 216, 268 MB 396 -> 419, 537 MB 881 -> 876; 288 bf16 tensors (1.9 GB written)
// 738 -> 690.  In place there is no difference.
bool grad_clip_streams(size_t bytes_written) { return bytes_written >= (size_t)384 << 20; }

template <int N> hipError_t grad_clip(const GradBatch<N> &b, const GradResult *result, bool stream, hipStream_t st) {
    if (stream) grad_clip_kernel<true, N><<<grad_norm_blocks(b), 256, 0, st>>>(b, result);
    else grad_clip_kernel<false, N><<<grad_norm_blocks(b), 256, 0, st>>>(b, result);
    return hipGetLastError();
}

#define INSTANTIATE(N) \
    template void grad_chunks(GradBatch<N> &); \
    template int grad_norm_blocks(const GradBatch<N> &); \
    template hipError_t grad_sum_sq(const GradBatch<N> &, double *, hipStream_t); \
    template hipError_t grad_clip(const GradBatch<N> &, const GradResult *, bool, hipStream_t);
INSTANTIATE(GRAD_BATCH)
INSTANTIATE(GRAD_FEW)
#undef INSTANTIATE

}  // namespace mmt
