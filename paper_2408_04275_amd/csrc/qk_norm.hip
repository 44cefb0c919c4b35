// Norms of query and key heads and their rotation in one pass; backward with the gains' gradients.
//
// A head belongs to a group of `lanes` threads of one wavefront (a power of two), each of which holds two chunks of V elements as in
// rope.hip: features that rotate with one another, so that only the head's sums go across lanes.  A workgroup takes whole tokens: first the
// rotations of its tokens go into LDS (an angle in fp64 each, reduced to a turn), then its threads walk over the query heads and then over the
// key heads, a kind's gains in registers.
#include "ops.h"
#include "chunk.h"
#include <algorithm>

namespace mmt {
namespace {

struct QkShape {
    int lanes;                  // threads a head
    int units, rot_units, copy_chunks;      // chunk pairs of a head: first the rotated ones, then those that pass through
    int tile;                   // tokens whose rotations are in LDS at a time
};

template <int V>
struct Place {                  // a thread's two chunks of a head
    int o0, o1;
    bool rotates, first, second;
    __device__ __forceinline__ Place(const QkShape &s, int half, int u) {
        rotates = u < s.rot_units;
        first = u < s.units;
        const int copy = u - s.rot_units, copy_units = s.units - s.rot_units;
        o0 = rotates ? u * V : 2 * half + copy * V;
        o1 = rotates ? o0 + half : o0 + copy_units * V;
        second = rotates || (first && copy + copy_units < s.copy_chunks);
    }
};

__device__ __forceinline__ float head_sum(float v, int lanes) {
    for (int o = 1; o < lanes; o *= 2) v += __shfl_xor(v, o, 64);
    return v;
}

// the rotations of tokens t0 .. t0 + tokens - 1, [tokens][half] (cosine, sine)
__device__ __forceinline__ void put_rotations(const RopeArgs &a, float2 *turned, int t0, int tokens) {
    for (int k = threadIdx.x; k < tokens * a.half; k += 256) {
        const int t = t0 + k / a.half;
        const int pos = a.positions ? a.positions[t] : t - a.cu[find_segment(a.cu, a.S, t)];
        const double turn = pos * a.turns[k % a.half];
        float si, co;
        sincospif(2.f * (float)(turn - rint(turn)), &si, &co);
        turned[k] = make_float2(co * a.cos_scale, si * a.sin_scale);
    }
}

template <int V, bool INTERLEAVED>
__device__ __forceinline__ void rotate(float (&lo)[V], float (&hi)[V], const float2 *cs, const Place<V> &p, int u) {
    auto turn = [](float &x, float &y, float2 r) {
        const float v = x;
        x = v * r.x - y * r.y;
        y = y * r.x + v * r.y;
    };
    if constexpr (INTERLEAVED) {
#pragma unroll
        for (int i = 0; i < V; i += 2) {
            turn(lo[i], lo[i + 1], cs[(p.o0 + i) / 2]);
            turn(hi[i], hi[i + 1], cs[(p.o1 + i) / 2]);
        }
    } else {
#pragma unroll
        for (int i = 0; i < V; ++i) turn(lo[i], hi[i], cs[u * V + i]);
    }
}

template <typename T, int V>
__device__ __forceinline__ void load_pair(const T *x, const Place<V> &p, float (&lo)[V], float (&hi)[V]) {
    Chunk<T, V> c0, c1;
    if (p.first) c0.load(x + p.o0);
    if (p.second) c1.load(x + p.o1);
#pragma unroll
    for (int i = 0; i < V; ++i) {
        lo[i] = p.first ? c0.get(i) : 0.f;
        hi[i] = p.second ? c1.get(i) : 0.f;
    }
}
template <typename T, int V>
__device__ __forceinline__ void store_pair(T *y, const Place<V> &p, const float (&lo)[V], const float (&hi)[V]) {
    Chunk<T, V> c0, c1;
    c0.set(lo);
    c1.set(hi);
    if (p.first) c0.store(y + p.o0);
    if (p.second) c1.store(y + p.o1);
}

// v -> (v - mean) rstd; returns rstd.  Chunks that a thread does not have are zero before and after.
template <int V, bool LAYER>
__device__ __forceinline__ float normalise(float (&lo)[V], float (&hi)[V], const Place<V> &p, int lanes, float inv_d, float eps) {
    if constexpr (LAYER) {
        float s = 0.f;
#pragma unroll
        for (int i = 0; i < V; ++i) s += lo[i] + hi[i];
        const float mean = head_sum(s, lanes) * inv_d;
#pragma unroll
        for (int i = 0; i < V; ++i) {
            lo[i] = p.first ? lo[i] - mean : 0.f;
            hi[i] = p.second ? hi[i] - mean : 0.f;
        }
    }
    float s = 0.f;
#pragma unroll
    for (int i = 0; i < V; ++i) s += lo[i] * lo[i] + hi[i] * hi[i];
    const float rstd = 1.f / sqrtf(head_sum(s, lanes) * inv_d + eps);
#pragma unroll
    for (int i = 0; i < V; ++i) { lo[i] *= rstd; hi[i] *= rstd; }
    return rstd;
}

template <typename T, int V, bool INTERLEAVED, bool LAYER>
__global__ __launch_bounds__(256) void qk_norm_fwd_kernel(QkNormArgs a, QkShape s) {
    extern __shared__ float2 turned[];
    const RopeArgs &r = a.r;
    const long first = (blockIdx.y * (long)gridDim.x + blockIdx.x) * s.tile;
    if (first >= r.T) return;
    const int t0 = (int)first, tokens = min(s.tile, r.T - t0);
    const int u = threadIdx.x & (s.lanes - 1), g = threadIdx.x / s.lanes, groups = 256 / s.lanes;
    const Place<V> p(s, r.half, u);
    const float inv_d = 1.f / r.d;
    put_rotations(r, turned, t0, tokens);
    __syncthreads();
    for (int kind = 0; kind < 2; ++kind) {
        const int h0 = kind ? a.nq : 0, heads = kind ? r.heads - a.nq : a.nq;
        if (!heads) continue;
        float w0[V], w1[V], b0[V], b1[V];
        load_pair((const T *)(kind ? a.k_w : a.q_w), p, w0, w1);
        if constexpr (LAYER) load_pair((const T *)(kind ? a.k_b : a.q_b), p, b0, b1);
        for (int i = g; i < tokens * heads; i += groups) {
            const int tok = i / heads, head = h0 + i % heads;
            float lo[V], hi[V];
            load_pair((const T *)r.x + (t0 + tok) * r.ldx + (long)head * r.d, p, lo, hi);
            normalise<V, LAYER>(lo, hi, p, s.lanes, inv_d, a.eps);
#pragma unroll
            for (int e = 0; e < V; ++e) {
                lo[e] = LAYER ? lo[e] * w0[e] + b0[e] : lo[e] * w0[e];
                hi[e] = LAYER ? hi[e] * w1[e] + b1[e] : hi[e] * w1[e];
            }
            if (p.rotates) rotate<V, INTERLEAVED>(lo, hi, turned + tok * r.half, p, u);
            store_pair((T *)r.y + (t0 + tok) * r.ldy + (long)head * r.d, p, lo, hi);
        }
    }
}

template <typename T, int V, bool INTERLEAVED, bool LAYER>
__global__ __launch_bounds__(256) void qk_norm_bwd_kernel(QkNormArgs a, QkShape s) {
    extern __shared__ float2 turned[];
    const RopeArgs &r = a.r;
    const int u = threadIdx.x & (s.lanes - 1), g = threadIdx.x / s.lanes, groups = 256 / s.lanes;
    const Place<V> p(s, r.half, u);
    const float inv_d = 1.f / r.d;
    float *const sums = (float *)turned;                     // [groups][d], when the rotations are done with
    for (int kind = 0; kind < 2; ++kind) {
        const int h0 = kind ? a.nq : 0, heads = kind ? r.heads - a.nq : a.nq;
        if (!heads) continue;
        float w0[V], w1[V], gw0[V], gw1[V], gb0[V], gb1[V];
        load_pair((const T *)(kind ? a.k_w : a.q_w), p, w0, w1);
#pragma unroll
        for (int e = 0; e < V; ++e) gw0[e] = gw1[e] = gb0[e] = gb1[e] = 0.f;
        for (long first = (long)blockIdx.x * s.tile; first < r.T; first += (long)gridDim.x * s.tile) {
            const int t0 = (int)first, tokens = min(s.tile, r.T - t0);
            __syncthreads();
            put_rotations(r, turned, t0, tokens);
            __syncthreads();
            for (int i = g; i < tokens * heads; i += groups) {
                const int tok = i / heads, head = h0 + i % heads;
                float lo[V], hi[V], d0[V], d1[V];
                load_pair((const T *)r.x + (t0 + tok) * r.ldx + (long)head * r.d, p, lo, hi);
                load_pair((const T *)a.dy + (t0 + tok) * a.lddy + (long)head * r.d, p, d0, d1);
                const float rstd = normalise<V, LAYER>(lo, hi, p, s.lanes, inv_d, a.eps);
                if (p.rotates) rotate<V, INTERLEAVED>(d0, d1, turned + tok * r.half, p, u);
                float dot = 0.f, mean = 0.f;
#pragma unroll
                for (int e = 0; e < V; ++e) {
                    gw0[e] += d0[e] * lo[e]; gw1[e] += d1[e] * hi[e];
                    if constexpr (LAYER) { gb0[e] += d0[e]; gb1[e] += d1[e]; }
                    d0[e] *= w0[e]; d1[e] *= w1[e];
                    dot += d0[e] * lo[e] + d1[e] * hi[e];
                    if constexpr (LAYER) mean += d0[e] + d1[e];
                }
                dot = head_sum(dot, s.lanes) * inv_d;
                if constexpr (LAYER) mean = head_sum(mean, s.lanes) * inv_d;
#pragma unroll
                for (int e = 0; e < V; ++e) {
                    d0[e] = rstd * (d0[e] - mean - lo[e] * dot);
                    d1[e] = rstd * (d1[e] - mean - hi[e] * dot);
                }
                if (r.y) store_pair((T *)r.y + (t0 + tok) * r.ldy + (long)head * r.d, p, d0, d1);
            }
        }
        for (int k = 0; k < (LAYER ? 2 : 1); ++k) {
            float *out = a.part[2 * kind + k];
            if (!out) continue;
            __syncthreads();
#pragma unroll
            for (int e = 0; e < V; ++e) {
                if (p.first) sums[g * r.d + p.o0 + e] = k ? gb0[e] : gw0[e];
                if (p.second) sums[g * r.d + p.o1 + e] = k ? gb1[e] : gw1[e];
            }
            __syncthreads();
            for (int f = threadIdx.x; f < r.d; f += 256) {
                float t = 0.f;
                for (int j = 0; j < groups; ++j) t += sums[j * r.d + f];
                out[(size_t)blockIdx.x * r.d + f] = t;
            }
        }
    }
}

template <int V> QkShape shape_of(const QkNormArgs &a) {
    QkShape s;
    s.rot_units = a.r.half / V;
    s.copy_chunks = (a.r.d - 2 * a.r.half) / V;
    s.units = s.rot_units + (s.copy_chunks + 1) / 2;         // at most 64
    s.lanes = 1;
    while (s.lanes < s.units) s.lanes *= 2;
    return s;
}

template <typename T, int V>
hipError_t launch(const QkNormArgs &a, bool back, hipStream_t st) {
    QkShape s = shape_of<V>(a);
    const int by_angles = a.r.half ? 1024 / a.r.half : 1024;
    const bool layer = a.norm == NORM_LAYER;
    if (back) {
        s.tile = std::max(1, std::min(by_angles, 16));
        const size_t lds = std::max((size_t)s.tile * a.r.half * sizeof(float2), (size_t)(256 / s.lanes) * a.r.d * sizeof(float));
        const int grid = qk_norm_bwd_blocks(a.r.T);
        if (a.r.interleaved) {
            if (layer) qk_norm_bwd_kernel<T, V, true, true><<<grid, 256, lds, st>>>(a, s);
            else qk_norm_bwd_kernel<T, V, true, false><<<grid, 256, lds, st>>>(a, s);
        } else if (layer) qk_norm_bwd_kernel<T, V, false, true><<<grid, 256, lds, st>>>(a, s);
        else qk_norm_bwd_kernel<T, V, false, false><<<grid, 256, lds, st>>>(a, s);
        return hipGetLastError();
    }
    const int by_units = (511 + a.r.heads * s.lanes) / (a.r.heads * s.lanes);
    s.tile = std::max(1, std::min({by_units, by_angles, a.r.T / 512}));
    const size_t lds = (size_t)s.tile * a.r.half * sizeof(float2);
    const int blocks = ceil_div(a.r.T, s.tile);
    const dim3 grid(std::min(blocks, 1 << 20), ceil_div(blocks, 1 << 20));
    if (a.r.interleaved) {
        if (layer) qk_norm_fwd_kernel<T, V, true, true><<<grid, 256, lds, st>>>(a, s);
        else qk_norm_fwd_kernel<T, V, true, false><<<grid, 256, lds, st>>>(a, s);
    } else if (layer) qk_norm_fwd_kernel<T, V, false, true><<<grid, 256, lds, st>>>(a, s);
    else qk_norm_fwd_kernel<T, V, false, false><<<grid, 256, lds, st>>>(a, s);
    return hipGetLastError();
}

hipError_t dispatch(int dtype, const QkNormArgs &a, bool back, hipStream_t st) {
    // the widest chunks that half and whole of a head are made of; rows and heads are 16 bytes apart
    const int half = a.r.half;
    if (dtype == DT_F32) return half % 4 == 0 ? launch<float, 4>(a, back, st) : launch<float, 2>(a, back, st);
    return half % 8 == 0 ? launch<bf16_t, 8>(a, back, st) : half % 4 == 0 ? launch<bf16_t, 4>(a, back, st) : launch<bf16_t, 2>(a, back, st);
}

}  // namespace

hipError_t qk_norm_fwd(int dtype, const QkNormArgs &a, hipStream_t st) { return a.r.T == 0 ? hipSuccess : dispatch(dtype, a, false, st); }

int qk_norm_bwd_blocks(int T) { return std::max(1, std::min(T, 1024)); }

hipError_t qk_norm_bwd(int dtype, const QkNormArgs &a, hipStream_t st) {
    if (a.r.T > 0) {
        const hipError_t e = dispatch(dtype, a, true, st);
        if (e != hipSuccess) return e;
    }
    const int rows = a.r.T > 0 ? qk_norm_bwd_blocks(a.r.T) : 0;
    ReduceJob jobs[4];
    for (int i = 0; i < 4; ++i) jobs[i] = {a.part[i], a.part[i] ? a.grad[i] : nullptr, rows, a.r.d};
    return reduce_jobs(a.grad_f32 ? DT_F32 : DT_BF16, jobs, 4, a.accumulate, st);
}

}  // namespace mmt
