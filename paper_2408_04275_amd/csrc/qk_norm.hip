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
    int step_tokens, step_heads;// heads that a workgroup has at work at once: step_tokens * heads + step_heads
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

// Sum over the head's lanes, the same in all of them; up to 16 lanes are added with DPP moves, which stay in the vector ALU
template <int CTRL> __device__ __forceinline__ float add_dpp(float v) { return v + __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), CTRL, 0xf, 0xf, false)); }
__device__ __forceinline__ float head_sum(float v, int lanes) {
    if (lanes > 1) v = add_dpp<0xb1>(v);            // quad_perm 1 0 3 2
    if (lanes > 2) v = add_dpp<0x4e>(v);            // quad_perm 2 3 0 1
    if (lanes > 4) v = add_dpp<0x141>(v);           // row_half_mirror
    if (lanes > 8) v = add_dpp<0x140>(v);           // row_mirror
    if (lanes > 16) v += __shfl_xor(v, 16, 64);
    if (lanes > 32) v += __shfl_xor(v, 32, 64);
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
struct Pair {                   // a thread's chunks as loaded
    Chunk<T, V> c0, c1;
    __device__ __forceinline__ void load(const T *x, const Place<V> &p) {
        if (p.first) c0.load(x + p.o0);
        if (p.second) c1.load(x + p.o1);
    }
    __device__ __forceinline__ void get(const Place<V> &p, float (&lo)[V], float (&hi)[V]) const {
#pragma unroll
        for (int i = 0; i < V; ++i) {
            lo[i] = p.first ? c0.get(i) : 0.f;
            hi[i] = p.second ? c1.get(i) : 0.f;
        }
    }
};
template <typename T, int V>
__device__ __forceinline__ void load_pair(const T *x, const Place<V> &p, float (&lo)[V], float (&hi)[V]) {
    Pair<T, V> c;
    c.load(x, p);
    c.get(p, lo, hi);
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

// gains (and biases) of both kinds in LDS, [2][d] each
template <typename T, bool LAYER>
__device__ __forceinline__ void put_gains(const QkNormArgs &a, float *gains) {
    const int d = a.r.d;
    for (int i = threadIdx.x; i < (LAYER ? 4 : 2) * d; i += 256) {
        const int k = i / d;
        const void *p = k == 0 ? a.q_w : k == 1 ? a.k_w : k == 2 ? a.q_b : a.k_b;
        gains[i] = p ? Elem<T>::load((const T *)p + i % d) : 0.f;
    }
}
template <int V>
__device__ __forceinline__ void get_gains(const float *g, const Place<V> &p, float (&lo)[V], float (&hi)[V]) {
#pragma unroll
    for (int i = 0; i < V; ++i) { lo[i] = 0.f; hi[i] = 0.f; }
    if (p.first) {
#pragma unroll
        for (int i = 0; i < V; ++i) lo[i] = g[p.o0 + i];
    }
    if (p.second) {
#pragma unroll
        for (int i = 0; i < V; ++i) hi[i] = g[p.o1 + i];
    }
}

// The first heads' rows are requested in front of everything else, and the next ones' in front of each turn's arithmetic.
template <typename T, int V, bool INTERLEAVED, bool LAYER>
__global__ __launch_bounds__(256) void qk_norm_fwd_kernel(QkNormArgs a, QkShape s) {
    extern __shared__ float2 turned[];
    const RopeArgs &r = a.r;
    float *const gains = (float *)(turned + s.tile * r.half);
    const long first = (blockIdx.y * (long)gridDim.x + blockIdx.x) * s.tile;
    if (first >= r.T) return;
    const int t0 = (int)first, tokens = min(s.tile, r.T - t0);
    const int u = threadIdx.x & (s.lanes - 1), g = threadIdx.x / s.lanes;
    const Place<V> p(s, r.half, u);
    const float inv_d = 1.f / r.d;
    int tok = g / r.heads, head = g % r.heads;
    Pair<T, V> next;
    auto request = [&] { next.load((const T *)r.x + (t0 + tok) * r.ldx + (long)head * r.d, p); };
    if (tok < tokens) request();
    put_gains<T, LAYER>(a, gains);
    put_rotations(r, turned, t0, tokens);
    __syncthreads();
    while (tok < tokens) {
        T *const y = (T *)r.y + (t0 + tok) * r.ldy + (long)head * r.d;
        const float2 *cs = turned + tok * r.half;
        const float *w = gains + (head < a.nq ? 0 : r.d);
        float lo[V], hi[V], w0[V], w1[V], b0[V], b1[V];
        const Pair<T, V> now = next;
        tok += s.step_tokens; head += s.step_heads;
        if (head >= r.heads) { head -= r.heads; ++tok; }
        if (tok < tokens) request();
        now.get(p, lo, hi);
        normalise<V, LAYER>(lo, hi, p, s.lanes, inv_d, a.eps);
        get_gains(w, p, w0, w1);
        if constexpr (LAYER) get_gains(w + 2 * r.d, p, b0, b1);
#pragma unroll
        for (int e = 0; e < V; ++e) {
            lo[e] = LAYER ? lo[e] * w0[e] + b0[e] : lo[e] * w0[e];
            hi[e] = LAYER ? hi[e] * w1[e] + b1[e] : hi[e] * w1[e];
        }
        if (p.rotates) rotate<V, INTERLEAVED>(lo, hi, cs, p, u);
        store_pair(y, p, lo, hi);
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
        const int step_tokens = groups / heads, step_heads = groups % heads;
        float w0[V], w1[V], gw0[V], gw1[V], gb0[V], gb1[V];
        load_pair((const T *)(kind ? a.k_w : a.q_w), p, w0, w1);
#pragma unroll
        for (int e = 0; e < V; ++e) gw0[e] = gw1[e] = gb0[e] = gb1[e] = 0.f;
        for (long first = (long)blockIdx.x * s.tile; first < r.T; first += (long)gridDim.x * s.tile) {
            const int t0 = (int)first, tokens = min(s.tile, r.T - t0);
            int tok = g / heads, head = g % heads;
            Pair<T, V> next_x, next_d;
            auto request = [&] {
                next_x.load((const T *)r.x + (t0 + tok) * r.ldx + (long)(h0 + head) * r.d, p);
                next_d.load((const T *)a.dy + (t0 + tok) * a.lddy + (long)(h0 + head) * r.d, p);
            };
            if (tok < tokens) request();
            __syncthreads();                                 // the last tile's rotations are done with
            put_rotations(r, turned, t0, tokens);
            __syncthreads();
            while (tok < tokens) {
                float lo[V], hi[V], d0[V], d1[V];
                next_x.get(p, lo, hi);
                next_d.get(p, d0, d1);
                const float2 *cs = turned + tok * r.half;
                T *const out = (T *)r.y + (t0 + tok) * r.ldy + (long)(h0 + head) * r.d;
                tok += step_tokens; head += step_heads;
                if (head >= heads) { head -= heads; ++tok; }
                if (tok < tokens) request();
                const float rstd = normalise<V, LAYER>(lo, hi, p, s.lanes, inv_d, a.eps);
                if (p.rotates) rotate<V, INTERLEAVED>(d0, d1, cs, p, u);
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
                if (r.y) store_pair(out, p, d0, d1);
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
    s.step_tokens = 256 / s.lanes / a.r.heads;
    s.step_heads = 256 / s.lanes % a.r.heads;
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
    const size_t lds = (size_t)s.tile * a.r.half * sizeof(float2) + (layer ? 4 : 2) * a.r.d * sizeof(float);
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

int qk_norm_bwd_blocks(int T) { return std::max(1, std::min(T, 512)); }

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
