// Norms of query and key heads and their rotation in one pass; backward with the gains' gradients.
//
// A head belongs to a group of `lanes` threads of one wavefront (a power of two), each of which holds two chunks of V elements as in
// rope.hip: features that rotate with one another, so that only the head's sums go across lanes.  A workgroup takes whole tokens: first the
// rotations of its tokens go into LDS (an angle in fp64 each, reduced to a turn), then its threads walk over the heads: forward over all, the gains in LDS, backward over those of
// one kind, its gains in registers.  Bound by memory: 16411 tokens of 72 heads of 128, LayerNorm, 120 us (5.0 TB/s), back 8192 of 64, RMSNorm, 86 (4.7) and 4 for the
// sums of the partial gains.
#include "ops.h"
#include "chunk.h"
#include <algorithm>

namespace mmt {
namespace {

struct QkShape {
    int lanes;                  // threads a head
    int units, rot_units, copy_chunks;      // chunk pairs of a head: first the rotated ones, then those that pass through
    int tile;                   // tokens whose rotations are in LDS at a time
    int q_blocks;               // backward: workgroups of the query heads
};

// Where a thread's two chunks of a head stand.  LANES: threads a head, where each of them has two chunks (4, 8 or 16); 0: any shape, and chunks that a
// thread does not have are those of unit 0, loaded to no purpose.
template <int V, int LANES>
struct Place {
    int o0, o1;
    bool rotates, first, second;
    __device__ __forceinline__ Place(const QkShape &s, int half, int u) {
        rotates = u < s.rot_units;
        const int copy = u - s.rot_units, copy_units = s.units - s.rot_units;
        first = LANES > 0 || u < s.units;
        second = LANES > 0 || rotates || (first && copy + copy_units < s.copy_chunks);
        o0 = !first ? 0 : rotates ? u * V : 2 * half + copy * V;
        o1 = !second ? 0 : rotates ? o0 + half : o0 + copy_units * V;
    }
};

// Sum over the head's lanes, the same in all of them; up to 16 lanes are added with DPP moves, which stay in the vector ALU
template <int CTRL> __device__ __forceinline__ float add_dpp(float v) { return v + __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), CTRL, 0xf, 0xf, false)); }
template <int LANES>
__device__ __forceinline__ float head_sum(float v, int lanes) {
    if constexpr (LANES > 0) lanes = LANES;
    if (lanes > 1) v = add_dpp<0xb1>(v);            // quad_perm 1 0 3 2
    if (lanes > 2) v = add_dpp<0x4e>(v);            // quad_perm 2 3 0 1
    if (lanes > 4) v = add_dpp<0x141>(v);           // row_half_mirror
    if (lanes > 8) v = add_dpp<0x140>(v);           // row_mirror
    if (lanes > 16) v += __shfl_xor(v, 16, 64);
    if (lanes > 32) v += __shfl_xor(v, 32, 64);
    return v;
}

// the rotations of tokens t0 .. t0 + tokens - 1, [tokens][half] (cosine, sine)
__device__ __forceinline__ int position_of(const RopeArgs &a, int t) { return a.positions ? a.positions[t] : t - a.cu[find_segment(a.cu, a.S, t)]; }
// pos: their positions in LDS (null: each thread looks for its own)
template <int THREADS>
__device__ __forceinline__ void put_rotations(const RopeArgs &a, float2 *turned, int t0, int tokens, const int *pos_in_lds) {
    for (int k = threadIdx.x; k < tokens * a.half; k += THREADS) {
        const int pos = pos_in_lds ? pos_in_lds[k / a.half] : position_of(a, t0 + k / a.half);
        const double turn = pos * a.turns[k % a.half];
        float si, co;
        sincospif(2.f * (float)(turn - rint(turn)), &si, &co);
        turned[k] = make_float2(co * a.cos_scale, si * a.sin_scale);
    }
}

template <int V, bool INTERLEAVED, int LANES>
__device__ __forceinline__ void rotate(float (&lo)[V], float (&hi)[V], const float2 *cs, const Place<V, LANES> &p, int u) {
    if (!p.rotates) return;
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

template <typename T, int V, int LANES>
struct Pair {                   // a thread's chunks as loaded
    Chunk<T, V> c0, c1;
    __device__ __forceinline__ void load(const T *x, const Place<V, LANES> &p) {
        c0.load(x + p.o0);
        c1.load(x + p.o1);
    }
    __device__ __forceinline__ void get(const Place<V, LANES> &p, float (&lo)[V], float (&hi)[V]) const {
#pragma unroll
        for (int i = 0; i < V; ++i) {
            lo[i] = p.first ? c0.get(i) : 0.f;
            hi[i] = p.second ? c1.get(i) : 0.f;
        }
    }
};
template <typename T, int V, int LANES>
__device__ __forceinline__ void store_pair(T *y, const Place<V, LANES> &p, const float (&lo)[V], const float (&hi)[V]) {
    Chunk<T, V> c0, c1;
    c0.set(lo);
    c1.set(hi);
    if (p.first) c0.store(y + p.o0);
    if (p.second) c1.store(y + p.o1);
}

// v -> (v - mean) rstd; returns rstd.  Chunks that a thread does not have are zero before and after.
template <int V, bool LAYER, int LANES>
__device__ __forceinline__ float normalise(float (&lo)[V], float (&hi)[V], const Place<V, LANES> &p, int lanes, float inv_d, float eps) {
    if constexpr (LAYER) {
        float s = 0.f;
#pragma unroll
        for (int i = 0; i < V; ++i) s += lo[i] + hi[i];
        const float mean = head_sum<LANES>(s, lanes) * inv_d;
#pragma unroll
        for (int i = 0; i < V; ++i) {
            lo[i] = p.first ? lo[i] - mean : 0.f;
            hi[i] = p.second ? hi[i] - mean : 0.f;
        }
    }
    float s = 0.f;
#pragma unroll
    for (int i = 0; i < V; ++i) s += lo[i] * lo[i] + hi[i] * hi[i];
    const float rstd = 1.f / sqrtf(head_sum<LANES>(s, lanes) * inv_d + eps);
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
template <int V, int LANES>
__device__ __forceinline__ void get_gains(const float *g, const Place<V, LANES> &p, float (&lo)[V], float (&hi)[V]) {
#pragma unroll
    for (int i = 0; i < V; ++i) { lo[i] = g[p.o0 + i]; hi[i] = g[p.o1 + i]; }
}

// The (token, head) pairs of a tile that a group of threads has, one after the other; behind the last a load ahead takes the gains, so that
// it needs no branch (with one the compiler waits for all loads on their way in each turn) and no memory (a pair of the tile once more: HBM reads an eighth
// to a quarter more, as rows that have been read do not stay in the cache).
struct Walk {
    int tok, head, tokens, heads, step_tokens, step_heads;
    __device__ __forceinline__ Walk(int g, int groups, int tokens_, int heads_)
        : tok(g / heads_), head(g % heads_), tokens(tokens_), heads(heads_), step_tokens(groups / heads_), step_heads(groups % heads_) {}
    __device__ __forceinline__ bool live() const { return tok < tokens; }
    __device__ __forceinline__ void next() {
        tok += step_tokens; head += step_heads;
        if (head >= heads) { head -= heads; ++tok; }
    }
    // the pair's features in rows ld apart, x being the tile's first; or d others
    template <typename T> __device__ __forceinline__ const T *at(const T *x, long ld, int d, const void *others) const {
        return live() ? x + tok * ld + (long)head * d : (const T *)others;
    }
};

// The first heads' rows are requested in front of everything else, and the next ones' in front of each turn's arithmetic, into the other of
// two sets of registers.
template <typename T, int V, bool INTERLEAVED, bool LAYER, int LANES>
__global__ __launch_bounds__(256) void qk_norm_fwd_kernel(QkNormArgs a, QkShape s) {
    extern __shared__ float2 turned[];
    const RopeArgs &r = a.r;
    float *const gains = (float *)(turned + s.tile * r.half);
    const long first = (blockIdx.y * (long)gridDim.x + blockIdx.x) * s.tile;
    if (first >= r.T) return;
    const int t0 = (int)first, tokens = min(s.tile, r.T - t0), lanes = LANES > 0 ? LANES : s.lanes;
    const int u = threadIdx.x & (lanes - 1);
    const Place<V, LANES> p(s, r.half, u);
    const float inv_d = 1.f / r.d;
    Walk w(threadIdx.x / lanes, 256 / lanes, tokens, r.heads);
    auto request = [&](Pair<T, V, LANES> &to) { to.load(w.at((const T *)r.x + t0 * r.ldx, r.ldx, r.d, a.nq ? a.q_w : a.k_w), p); };
    auto turn = [&](const Pair<T, V, LANES> &now, Pair<T, V, LANES> &next) {
        T *const y = (T *)r.y + (t0 + w.tok) * r.ldy + (long)w.head * r.d;
        const float2 *cs = turned + w.tok * r.half;
        const float *gain = gains + (w.head < a.nq ? 0 : r.d);
        w.next();
        request(next);
        float lo[V], hi[V], w0[V], w1[V], b0[V], b1[V];
        now.get(p, lo, hi);
        normalise<V, LAYER>(lo, hi, p, lanes, inv_d, a.eps);
        get_gains(gain, p, w0, w1);
        if constexpr (LAYER) get_gains(gain + 2 * r.d, p, b0, b1);
#pragma unroll
        for (int e = 0; e < V; ++e) {
            lo[e] = LAYER ? lo[e] * w0[e] + b0[e] : lo[e] * w0[e];
            hi[e] = LAYER ? hi[e] * w1[e] + b1[e] : hi[e] * w1[e];
        }
        rotate<V, INTERLEAVED>(lo, hi, cs, p, u);
        store_pair(y, p, lo, hi);
    };
    Pair<T, V, LANES> even, odd;
    request(even);
    put_gains<T, LAYER>(a, gains);
    put_rotations<256>(r, turned, t0, tokens, nullptr);
    __syncthreads();
    while (w.live()) {
        turn(even, odd);
        if (!w.live()) break;
        turn(odd, even);
    }
}

// A workgroup has heads of one kind, of every so many tiles of tokens: query heads the first s.q_blocks, key heads the others.  Sixteen wavefronts a
// compute unit, in two workgroups of 512 threads: smaller ones would leave more partial rows, whose sum is a launch of its own.  The LayerNorm needs more than the
// 128 registers that leaves (8192 tokens of 72 heads: 163 us with 28 of them in memory): twelve wavefronts in three workgroups.
template <bool LAYER> constexpr int BWD_THREADS = LAYER ? 256 : 512;
template <bool LAYER> constexpr int BWD_BLOCKS = LAYER ? 768 : 512;
constexpr int BWD_TILE = 64;
template <typename T, int V, bool INTERLEAVED, bool LAYER, int LANES>
__global__ __launch_bounds__(BWD_THREADS<LAYER>, LAYER ? 3 : 4) void qk_norm_bwd_kernel(QkNormArgs a, QkShape s) {
    extern __shared__ float2 turned[];
    constexpr int THREADS = BWD_THREADS<LAYER>;
    const RopeArgs &r = a.r;
    const int lanes = LANES > 0 ? LANES : s.lanes;
    const int u = threadIdx.x & (lanes - 1), g = threadIdx.x / lanes, groups = THREADS / lanes;
    const Place<V, LANES> p(s, r.half, u);
    const float inv_d = 1.f / r.d;
    float *const sums = (float *)(turned + s.tile * r.half);  // [wavefronts][d]
    __shared__ int positions[BWD_TILE];
    const int kind = (int)blockIdx.x >= s.q_blocks, block = kind ? blockIdx.x - s.q_blocks : blockIdx.x, blocks = kind ? gridDim.x - s.q_blocks : s.q_blocks;
    const int h0 = kind ? a.nq : 0, heads = kind ? r.heads - a.nq : a.nq;
    Pair<T, V, LANES> gain;
    gain.load((const T *)(kind ? a.k_w : a.q_w), p);
    float w0[V], w1[V], gw0[V], gw1[V], gb0[V], gb1[V];
    gain.get(p, w0, w1);
#pragma unroll
    for (int e = 0; e < V; ++e) gw0[e] = gw1[e] = gb0[e] = gb1[e] = 0.f;
    for (long first = (long)block * s.tile; first < r.T; first += (long)blocks * s.tile) {
        const int t0 = (int)first, tokens = min(s.tile, r.T - t0);
        Walk w(g, groups, tokens, heads);
        struct Rows { Pair<T, V, LANES> x, d; } even, odd;
        auto request = [&](Rows &to) {
            const void *const others = kind ? a.k_w : a.q_w;
            to.x.load(w.at((const T *)r.x + t0 * r.ldx + (long)h0 * r.d, r.ldx, r.d, others), p);
            to.d.load(w.at((const T *)a.dy + t0 * a.lddy + (long)h0 * r.d, a.lddy, r.d, others), p);
        };
        auto turn = [&](const Rows &now, Rows &next) {
            const float2 *cs = turned + w.tok * r.half;
            T *const out = (T *)r.y + (t0 + w.tok) * r.ldy + (long)(h0 + w.head) * r.d;
            w.next();
            request(next);
            float lo[V], hi[V], d0[V], d1[V];
            now.x.get(p, lo, hi);
            now.d.get(p, d0, d1);
            const float rstd = normalise<V, LAYER>(lo, hi, p, lanes, inv_d, a.eps);
            rotate<V, INTERLEAVED>(d0, d1, cs, p, u);
            float dot = 0.f, mean = 0.f;
#pragma unroll
            for (int e = 0; e < V; ++e) {
                gw0[e] += d0[e] * lo[e]; gw1[e] += d1[e] * hi[e];
                if constexpr (LAYER) { gb0[e] += d0[e]; gb1[e] += d1[e]; }
                d0[e] *= w0[e]; d1[e] *= w1[e];
                dot += d0[e] * lo[e] + d1[e] * hi[e];
                if constexpr (LAYER) mean += d0[e] + d1[e];
            }
            dot = head_sum<LANES>(dot, lanes) * inv_d;
            if constexpr (LAYER) mean = head_sum<LANES>(mean, lanes) * inv_d;
#pragma unroll
            for (int e = 0; e < V; ++e) {
                d0[e] = rstd * (d0[e] - mean - lo[e] * dot);
                d1[e] = rstd * (d1[e] - mean - hi[e] * dot);
            }
            if (r.y) store_pair(out, p, d0, d1);
        };
        request(even);
        __syncthreads();                                 // the last tile's rotations are done with
        if (r.half && (int)threadIdx.x < tokens) positions[threadIdx.x] = position_of(r, t0 + threadIdx.x);
        __syncthreads();
        put_rotations<THREADS>(r, turned, t0, tokens, positions);
        __syncthreads();
        while (w.live()) {
            turn(even, odd);
            if (!w.live()) break;
            turn(odd, even);
        }
    }
    // the heads of a wavefront, then the wavefronts
    auto fold = [&](float (&v)[V]) {
        for (int o = lanes; o < 64; o *= 2)
#pragma unroll
            for (int e = 0; e < V; ++e) v[e] += __shfl_xor(v[e], o, 64);
    };
    for (int k = 0; k < (LAYER ? 2 : 1); ++k) {
        float *out = a.part[2 * kind + k];
        if (!out) continue;
        if (k) { fold(gb0); fold(gb1); }
        else { fold(gw0); fold(gw1); }
        __syncthreads();
        if ((int)(threadIdx.x & 63) < lanes) {
            float *mine = sums + (threadIdx.x >> 6) * r.d;
#pragma unroll
            for (int e = 0; e < V; ++e) {
                if (p.first) mine[p.o0 + e] = k ? gb0[e] : gw0[e];
                if (p.second) mine[p.o1 + e] = k ? gb1[e] : gw1[e];
            }
        }
        __syncthreads();
        for (int f = threadIdx.x; f < r.d; f += THREADS) {
            float t = 0.f;
#pragma unroll
            for (int j = 0; j < THREADS / 64; ++j) t += sums[j * r.d + f];
            out[(size_t)block * r.d + f] = t;
        }
    }
}

// workgroups of the backward pass: of the query heads, and of all; work as the heads are
int bwd_blocks(int T, bool layer) { return (int)std::max(1l, std::min(2l * T, (long)(layer ? BWD_BLOCKS<true> : BWD_BLOCKS<false>))); }
int bwd_q_blocks(const QkNormArgs &a) {
    const int all = bwd_blocks(a.r.T, a.norm == NORM_LAYER);
    if (!a.nq || a.nq == a.r.heads) return a.nq ? all : 0;
    return std::min(std::max((int)((long)all * a.nq / a.r.heads), 1), all - 1);
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

template <typename T, int V, bool INTERLEAVED, bool LAYER, int LANES>
hipError_t launch(const QkNormArgs &a, QkShape s, bool back, hipStream_t st) {
    const int by_angles = a.r.half ? 1024 / a.r.half : 1024;
    if (back) {
        const int all = bwd_blocks(a.r.T, LAYER);
        s.q_blocks = bwd_q_blocks(a);
        s.tile = std::max(1, std::min({2 * by_angles, BWD_TILE, ceil_div(a.r.T, std::max(s.q_blocks, all - s.q_blocks))}));
        const size_t lds = (size_t)s.tile * a.r.half * sizeof(float2) + (size_t)(BWD_THREADS<LAYER> / 64) * a.r.d * sizeof(float);
        qk_norm_bwd_kernel<T, V, INTERLEAVED, LAYER, LANES><<<all, BWD_THREADS<LAYER>, lds, st>>>(a, s);
        return hipGetLastError();
    }
    // Four turns a thread: with fewer the load behind the last is felt, with more the workgroups end apart.  us, 1 / 2 / 4 / 8 tokens a workgroup: 16411 tokens of
    // 72 heads of 128 134 / 125 / 129 / 135, 9536 of 32 of 64 21.3 / 20.0 / 17.7 / 17.0.
    const int by_units = (1023 + a.r.heads * s.lanes) / (a.r.heads * s.lanes);
    s.tile = std::max(1, std::min({by_units, by_angles, a.r.T / 512}));
    const size_t lds = (size_t)s.tile * a.r.half * sizeof(float2) + (LAYER ? 4 : 2) * a.r.d * sizeof(float);
    const int blocks = ceil_div(a.r.T, s.tile);
    const dim3 grid(std::min(blocks, 1 << 20), ceil_div(blocks, 1 << 20));
    qk_norm_fwd_kernel<T, V, INTERLEAVED, LAYER, LANES><<<grid, 256, lds, st>>>(a, s);
    return hipGetLastError();
}

template <typename T, int V, bool INTERLEAVED, bool LAYER>
hipError_t by_lanes(const QkNormArgs &a, bool back, hipStream_t st) {
    const QkShape s = shape_of<V>(a);
    if constexpr (V * sizeof(T) == 16)
        if (s.copy_chunks % 2 == 0 && s.units == s.lanes) {  // heads of 64, 128 or 256, however much of them rotates
            if (s.lanes == 4) return launch<T, V, INTERLEAVED, LAYER, 4>(a, s, back, st);
            if (s.lanes == 8) return launch<T, V, INTERLEAVED, LAYER, 8>(a, s, back, st);
            if (s.lanes == 16) return launch<T, V, INTERLEAVED, LAYER, 16>(a, s, back, st);
        }
    return launch<T, V, INTERLEAVED, LAYER, 0>(a, s, back, st);
}

template <typename T, int V>
hipError_t launch(const QkNormArgs &a, bool back, hipStream_t st) {
    const bool layer = a.norm == NORM_LAYER;
    if (a.r.interleaved) return layer ? by_lanes<T, V, true, true>(a, back, st) : by_lanes<T, V, true, false>(a, back, st);
    return layer ? by_lanes<T, V, false, true>(a, back, st) : by_lanes<T, V, false, false>(a, back, st);
}

hipError_t dispatch(int dtype, const QkNormArgs &a, bool back, hipStream_t st) {
    // the widest chunks that half and whole of a head are made of; rows and heads are 16 bytes apart
    const int half = a.r.half;
    if (dtype == DT_F32) return half % 4 == 0 ? launch<float, 4>(a, back, st) : launch<float, 2>(a, back, st);
    return half % 8 == 0 ? launch<bf16_t, 8>(a, back, st) : half % 4 == 0 ? launch<bf16_t, 4>(a, back, st) : launch<bf16_t, 2>(a, back, st);
}

}  // namespace

hipError_t qk_norm_fwd(int dtype, const QkNormArgs &a, hipStream_t st) { return a.r.T == 0 ? hipSuccess : dispatch(dtype, a, false, st); }

int qk_norm_bwd_blocks(int T, int norm) { return bwd_blocks(T, norm == NORM_LAYER); }

hipError_t qk_norm_bwd(int dtype, const QkNormArgs &a, hipStream_t st) {
    if (a.r.T > 0) {
        const hipError_t e = dispatch(dtype, a, true, st);
        if (e != hipSuccess) return e;
    }
    const int q_rows = a.r.T > 0 ? bwd_q_blocks(a) : 0, k_rows = a.r.T > 0 ? bwd_blocks(a.r.T, a.norm == NORM_LAYER) - q_rows : 0;
    ReduceJob jobs[4];
    for (int i = 0; i < 4; ++i) jobs[i] = {a.part[i], a.part[i] ? a.grad[i] : nullptr, i < 2 ? q_rows : k_rows, a.r.d};
    return reduce_jobs(a.grad_f32 ? DT_F32 : DT_BF16, jobs, 4, a.accumulate, st);
}

}  // namespace mmt
