// The join of a block's branch with the residual stream: norm behind the block, gate, scales, norm in front of the next.
//     n = norm_post(b);  y = alpha x + beta gate n;  h = norm_pre(y)
//
// Memory-bound: forward reads x and b and writes y and h, backward reads dy, dh, y and b and writes dx and db, each once; a row stays in
// registers from its first use to its last.  A row is worked on by a group of G threads with MC chunks of 8 columns each, and a
// workgroup of NT threads walks over a contiguous range of rows, NT / G at a time, the next ones requested before the present ones are
// reduced.  Gains, biases and gates stay in registers; so do backward's sums over tokens, which leave the workgroup as one partial row.
// Not every instance keeps these requests on their way while it works.  Backward does in bf16; in fp32 the compiler waits inside each turn for the statistics and
// rows just requested (4111 x 1280, two LayerNorms and segment gates 42 to 45 us for 25 us of bytes; where rows are wide it costs little, 9000 x 5120, two
// RMSNorms 230 for 221).  Forward with one chunk a thread does without a gate; with one, per channel too, it waits for the next row where the branch that loads a
// segment's gate joins (9000 bf16 rows of 1280, two LayerNorms: no gate 19.7 us, channel 22.7, segment 23.3; bytes 18.4).
// 8192 rows of 4096 in bf16, two RMSNorms: forward 55 us (4.9 TB/s), backward 81 us (4.9 TB/s) and 5 us for the sums of the partial rows; a copy
// of as many bytes runs at 5.0 to 5.4 TB/s.  Below about 2000 rows the launches and the first row's way through the chip bound both.
#include "ops.h"
#include "reduce.h"
#include "vec8.h"
#include "resident.h"
#include <algorithm>
#include <type_traits>

namespace mmt {
namespace {

// first row of workgroup b: the first T % blocks workgroups have one row more
__device__ __forceinline__ int join_row(int T, int blocks, int b) { return b * (T / blocks) + min(b, T % blocks); }

// find_segment for a token that is the same in all lanes: 64 boundaries are looked at together, so up to 64 segments take one load's time instead of
// one per halving
__device__ __forceinline__ int find_segment_wave(const int *cu, int S, int t) {
    int lo = 0, hi = S;
    while (hi - lo > 1) {
        const int step = (hi - lo + 63) >> 6, at = lo + (int)(threadIdx.x & 63) * step;
        lo += max(__popcll(__ballot(at < hi && cu[min(at, S)] <= t)) - 1, 0) * step;    // (cu[lo] <= t always)
        hi = min(hi, lo + step);
    }
    return lo;
}

// Sum over the wavefront, the same in all lanes.  Lanes are added with DPP moves, which stay in the vector ALU: with shuffles, each of which
// goes through the LDS unit, a row's sums were a chain of 6 x 100 clocks.  Quads, half rows and rows of 16 lanes are folded by permutations,
// then rows 0 and 2 are added to 1 and 3, and row 1 to 3.
template <int CTRL, int ROWS> __device__ __forceinline__ float add_dpp(float v) {
    return v + __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), CTRL, ROWS, 0xf, false));
}
__device__ __forceinline__ float wave_total(float v) {
    v = add_dpp<0xb1, 0xf>(v);          // quad_perm 1 0 3 2
    v = add_dpp<0x4e, 0xf>(v);          // quad_perm 2 3 0 1
    v = add_dpp<0x141, 0xf>(v);         // row_half_mirror
    v = add_dpp<0x140, 0xf>(v);         // row_mirror
    v = add_dpp<0x142, 0xa>(v);         // row_bcast 15 to rows 1 and 3
    v = add_dpp<0x143, 0xc>(v);         // row_bcast 31 to rows 2 and 3
    return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v), 63));
}

// Sums over the G threads of a row, MC chunks of 8 columns each.  red: two buffers, used in turn, so that one barrier per sum is enough (a
// thread that writes a buffer again has passed the barrier behind its last reading).  All threads of the workgroup call it together.
template <int G, int MC, int NT> struct RowSum {
    float2 (*red)[NT / 64];
    int H, turn = 0;
    __device__ __forceinline__ void operator()(float &a, float &b) {
        a = wave_total(a); b = wave_total(b);
        if constexpr (G > 64) {
            const float2 *all = share(make_float2(a, b));
            a = b = 0.f;
#pragma unroll
            for (int i = 0; i < G / 64; ++i) { a += all[i].x; b += all[i].y; }
        }
    }
    __device__ __forceinline__ void operator()(float &a) {
        a = wave_total(a);
        if constexpr (G > 64) {
            const float2 *all = share(make_float2(a, 0.f));
            a = 0.f;
#pragma unroll
            for (int i = 0; i < G / 64; ++i) a += all[i].x;
        }
    }
    __device__ __forceinline__ const float2 *share(float2 mine) {
        if ((threadIdx.x & 63) == 0) red[turn][threadIdx.x >> 6] = mine;
        __syncthreads();
        const float2 *all = &red[turn][threadIdx.x / G * (G / 64)];
        turn ^= 1;
        return all;
    }
    // columns of wavefront i of the row
    __device__ __forceinline__ float columns(int i) const {
        int n = 0;
#pragma unroll
        for (int k = 0; k < MC; ++k) n += min(max(H - (i * 64 + k * G) * 8, 0), 512);
        return (float)n;
    }
    // Mean and 1 / deviation of the row of which this thread holds v, zero outside of it.  MEAN: with the mean, if `layer` (zero otherwise), first
    // about each wavefront's own mean, then joined, so that nothing cancels however far the row is from zero and one barrier is enough.
    // inv_columns: 1 / the columns of this wavefront (0 if it has none).
    template <bool MEAN, typename In>
    __device__ __forceinline__ void statistics(const float (&v)[MC][8], bool layer, float inv_columns, float eps, In inside, float &mu, float &r) {
        const float inv_h = 1.f / H;
        float q = 0.f;
        mu = 0.f;
        if constexpr (MEAN) {
            float sum = 0.f;
#pragma unroll
            for (int i = 0; i < MC; ++i)
#pragma unroll
                for (int j = 0; j < 8; ++j) sum += v[i][j];
            sum = wave_total(sum) * inv_columns;
            mu = layer ? sum : 0.f;
        }
#pragma unroll
        for (int i = 0; i < MC; ++i) {
            float t = 0.f;
#pragma unroll
            for (int j = 0; j < 8; ++j) t += (v[i][j] - mu) * (v[i][j] - mu);
            q += !MEAN || inside(i) ? t : 0.f;
        }
        q = wave_total(q);
        if constexpr (G > 64) {
            const float2 *all = share(make_float2(mu, q));
            q = mu = 0.f;
            if constexpr (MEAN) {
#pragma unroll
                for (int i = 0; i < G / 64; ++i) mu += columns(i) * all[i].x;
                mu *= inv_h;
#pragma unroll
                for (int i = 0; i < G / 64; ++i) q += all[i].y + columns(i) * (all[i].x - mu) * (all[i].x - mu);
            } else {
#pragma unroll
                for (int i = 0; i < G / 64; ++i) q += all[i].y;
            }
        }
        r = rsqrtf(q * inv_h + eps);
    }
};

__device__ __forceinline__ f32x4 load4(const float *p) { return *reinterpret_cast<const f32x4 *>(p); }
__device__ __forceinline__ f32x4 load4(const bf16_t *p) {
    const u32x2 r = *reinterpret_cast<const u32x2 *>(p);
    return {__uint_as_float(r[0] << 16), __uint_as_float(r[0] & 0xffff0000u), __uint_as_float(r[1] << 16), __uint_as_float(r[1] & 0xffff0000u)};
}
__device__ __forceinline__ void store4(float *p, f32x4 v) { *reinterpret_cast<f32x4 *>(p) = v; }
__device__ __forceinline__ void store4(bf16_t *p, f32x4 v) { *reinterpret_cast<u32x2 *>(p) = u32x2{pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3])}; }

template <typename T> __device__ __forceinline__ void zero8(Raw8<T> &r) { __builtin_memset(&r, 0, sizeof(r)); }

// LN: one of the norms is a LayerNorm (gains only otherwise); the other may be an RMSNorm, which then has mean and bias zero.
template <typename T, int G, int MC, int NT, bool LN, bool GATE, bool POST>
__global__ __launch_bounds__(NT, sizeof(T) == 2 && MC > 1 ? 4 : 1) void join_fwd_kernel(JoinArgs a) {
    constexpr int R = NT / G;
    constexpr bool IN_LDS = LN && MC > 1 && G > 256 && sizeof(T) == 2;
    __shared__ float2 red[2][NT / 64];
    // a wavefront has one row's columns: rows are scalars, and addresses a scalar and a column
    const int lane = threadIdx.x % G, grp = __builtin_amdgcn_readfirstlane(threadIdx.x / G), H = a.H;
    RowSum<G, MC, NT> row_sum{red, H};
    const int r0 = join_row(a.T, gridDim.x, blockIdx.x), r1 = join_row(a.T, gridDim.x, blockIdx.x + 1);
    const float wave_columns = row_sum.columns(__builtin_amdgcn_readfirstlane(lane / 64)), inv_columns = wave_columns > 0.f ? 1.f / wave_columns : 0.f;
    auto col = [&](int i) { return (lane + i * G) * 8; };
    auto inside = [&](int i) { return col(i) < H; };
    // IN_LDS: gains and biases wait in LDS, each thread's own, where registers for them would cost a workgroup per compute unit (9000 rows of
    // 8192, two LayerNorms and a gate: 205 -> 152 us)
    __shared__ __attribute__((aligned(16))) T parked[IN_LDS ? 4 : 1][IN_LDS ? G * MC * 8 : 8];
    constexpr int HELD = IN_LDS ? 1 : MC;
    Raw8<T> nx[MC], nb[MC], w1[HELD], w2[POST ? HELD : 1], b1[LN ? HELD : 1], b2[LN && POST ? HELD : 1], gt[GATE ? MC : 1];
    // a parameter's chunk; zero where there is none, so that what is outside of the row stays zero throughout
    auto keep = [&](Raw8<T> *held, int slot, int i, const void *from) {
        Raw8<T> v;
        zero8(v);
        if (from && inside(i)) v = load_plain8((const T *)from + col(i));
        if constexpr (IN_LDS) *reinterpret_cast<Raw8<T> *>(&parked[slot][col(i)]) = v;
        else held[i] = v;
    };
    auto kept = [&](Raw8<T> *held, int slot, int i) {
        if constexpr (IN_LDS) return *reinterpret_cast<const Raw8<T> *>(&parked[slot][col(i)]);
        else return held[i];
    };
#pragma unroll
    for (int i = 0; i < MC; ++i) { zero8(nx[i]); zero8(nb[i]); }
    auto request = [&](int row) {
        if (row >= r1) return;
#pragma unroll
        for (int i = 0; i < MC; ++i) {
            if (!inside(i)) continue;
            const size_t at = (size_t)row * H + col(i);
            load_raw8((const T *)a.x + at, nx[i]);
            if (a.b) load_raw8((const T *)a.b + at, nb[i]);
        }
    };
    request(r0 + grp);
#pragma unroll
    for (int i = 0; i < MC; ++i) {
        keep(w1, 0, i, a.pre_w);
        if constexpr (LN) keep(b1, 1, i, a.pre_b);
        if constexpr (POST) keep(w2, 2, i, a.post_w);
        if constexpr (LN && POST) keep(b2, 3, i, a.post_b);
        if constexpr (GATE) {
            zero8(gt[i]);
            if (a.gate == GATE_CHANNEL && inside(i)) gt[i] = load_plain8((const T *)a.gate_v + col(i));
        }
    }
    int seg_end = 0;
    // v <- normalised v, gain and bias applied
    auto norm = [&](float (&v)[MC][8], bool layer, float eps, Raw8<T> *w, Raw8<T> *bias, int slot, float &mu, float &r) {
        row_sum.template statistics<LN>(v, layer, inv_columns, eps, inside, mu, r);
#pragma unroll
        for (int i = 0; i < MC; ++i) {
            float g[8], o[8];
            unpack8(kept(w, slot, i), g);
            if constexpr (LN) unpack8(kept(bias, slot + 1, i), o);
#pragma unroll
            for (int j = 0; j < 8; ++j) v[i][j] = (v[i][j] - mu) * r * g[j] + (LN ? o[j] : 0.f);
        }
    };
    for (int base = r0; base < r1; base += R) {
        const int row = base + grp;
        const bool valid = row < r1;
        float v[MC][8], n[MC][8], mu, r;
#pragma unroll
        for (int i = 0; i < MC; ++i) { unpack8(nx[i], v[i]); unpack8(nb[i], n[i]); }
        request(row + R);
        if (a.b) {
            if constexpr (GATE) {
                if (a.gate == GATE_SEGMENT && valid && row >= seg_end) {
                    const int seg = find_segment_wave(a.cu, a.S, row);
                    seg_end = a.cu[seg + 1];
#pragma unroll
                    for (int i = 0; i < MC; ++i)
                        if (inside(i)) gt[i] = load_plain8((const T *)a.gate_v + (size_t)seg * H + col(i));
                }
            }
            if constexpr (POST) {
                norm(n, a.post == NORM_LAYER, a.post_eps, w2, b2, 2, mu, r);
                if (lane == 0 && valid) {
                    if (a.post_rstd) a.post_rstd[row] = r;
                    if (LN && a.post == NORM_LAYER && a.post_mean) a.post_mean[row] = mu;
                }
            }
#pragma unroll
            for (int i = 0; i < MC; ++i) {
                float g[8];
                if constexpr (GATE) unpack8(gt[i], g);
#pragma unroll
                for (int j = 0; j < 8; ++j) v[i][j] = a.alpha * v[i][j] + a.beta * (GATE ? g[j] * n[i][j] : n[i][j]);
                if (valid && inside(i)) store8((T *)a.y + (size_t)row * H + col(i), v[i]);
            }
        }
        if (a.pre == NORM_NONE) continue;
        norm(v, a.pre == NORM_LAYER, a.pre_eps, w1, b1, 0, mu, r);
        if (lane == 0 && valid) {
            if (a.pre_rstd) a.pre_rstd[row] = r;
            if (LN && a.pre == NORM_LAYER && a.pre_mean) a.pre_mean[row] = mu;
        }
#pragma unroll
        for (int i = 0; i < MC; ++i)
            if (valid && inside(i)) store8((T *)a.h + (size_t)row * H + col(i), v[i]);
    }
}

// With hat = (v - mean) r and back = d_out w, a norm's input gradient is r (back - mean(back) [LAYER] - hat mean(back hat)); gain and bias
// get sum d_out hat and sum d_out.  Gradient of y: d = dy + the pre norm's; then dx = alpha d, and the branch gets beta gate d through the
// post norm.  A gate is the same in all rows of its segment (or in all rows), so the sums A = sum d hat and B = sum d over these rows give all three
// gradients behind the block: gain beta gate A, bias beta gate B, gate beta (w A + b B), or beta A with hat = branch where there is no post norm.
//
// By segment, a workgroup's gate sums go out at the end of each segment's rows: as the gradient where it has all of them, else into its
// slot 0 if its range begins inside the segment or with it, and into slot 1 otherwise (then the range ends in it); the post norm's sums are added up in
// LDS.  One workgroup per compute unit: more leave more partial rows to be added up (two RMSNorms in bf16, 256, 512 and 1024 workgroups: 9000 rows of 1280
// 41.5, 44.5, 52.9 us, 600 rows of 8192 23.4, 32.1, 34.3; only rows of up to 512 would gain by two, 22.1 and 19.8).
template <typename T, int G, int MC, int NT, bool LN, bool GATE, bool POST>
__global__ __launch_bounds__(NT) void join_bwd_kernel(JoinArgs a) {
    constexpr int R = NT / G, W = G * MC * 8;
    constexpr bool SUM_A = POST || GATE, SUM_B = LN && POST;
    constexpr bool IN_LDS = LN && POST && MC > 1 && (GATE || sizeof(T) == 4);
    __shared__ float2 red[2][NT / 64];
    __shared__ __attribute__((aligned(16))) float comb[LN ? 2 : 1][R > 1 ? R : 1][R > 1 ? W : 4];
    __shared__ __attribute__((aligned(16))) float total_w[GATE && POST ? W : 4], total_b[GATE && SUM_B ? W : 4];
    const int lane = threadIdx.x % G, grp = __builtin_amdgcn_readfirstlane(threadIdx.x / G), H = a.H, block = blockIdx.x;
    RowSum<G, MC, NT> row_sum{red, H};
    const int r0 = join_row(a.T, gridDim.x, block), r1 = join_row(a.T, gridDim.x, block + 1);
    const float inv_h = 1.f / H;
    const bool pre = a.pre != NORM_NONE, by_segment = GATE && a.gate == GATE_SEGMENT;
    auto col = [&](int i) { return (lane + i * G) * 8; };
    auto inside = [&](int i) { return col(i) < H; };
    const float alpha = a.b ? a.alpha : 1.f;
    // IN_LDS: the gains wait in LDS, each thread's own, where the kernel would spill most (9000 rows of 8192 in fp32, two LayerNorms and
    // a gate: 645 -> 420 us).  Registers that still spill, with a gate and a post norm: two LayerNorms in fp32 2, 2, 6 and 16 at 128, 192, 256 and 640 threads a row, 57
    // at 512 with two chunks (8 without the post norm), in bf16 2 at 640; two RMSNorms in fp32 14 at 512 with two chunks.
    __shared__ __attribute__((aligned(16))) T parked[IN_LDS ? 2 : 1][IN_LDS ? W : 8];
    constexpr int HELD = IN_LDS ? 1 : MC;
    Raw8<T> pdy[MC], pdh[MC], py[MC], pb[MC], w1[HELD], w2[POST ? HELD : 1], gt[GATE ? MC : 1];
    // a parameter's chunk; zero outside of the row, which keeps what is computed there out of the row's sums
    auto keep = [&](Raw8<T> *held, int slot, int i, const void *from) {
        Raw8<T> v;
        zero8(v);
        if (from && inside(i)) v = load_plain8((const T *)from + col(i));
        if constexpr (IN_LDS) *reinterpret_cast<Raw8<T> *>(&parked[slot][col(i)]) = v;
        else held[i] = v;
    };
    auto kept = [&](Raw8<T> *held, int slot, int i) {
        if constexpr (IN_LDS) return *reinterpret_cast<const Raw8<T> *>(&parked[slot][col(i)]);
        else return held[i];
    };
    float s_pre_w[MC][8] = {}, s_pre_b[LN ? MC : 1][8] = {}, sum_a[MC][8] = {}, sum_b[LN ? MC : 1][8] = {};
    float pr = 0.f, pmu = 0.f, pr2 = 0.f, pmu2 = 0.f;
#pragma unroll
    for (int i = 0; i < MC; ++i) { zero8(pdy[i]); zero8(pdh[i]); zero8(py[i]); zero8(pb[i]); }
    auto forget = [&] {                         // no row: adds nothing to any sum
        pr = pmu = pr2 = pmu2 = 0.f;
#pragma unroll
        for (int i = 0; i < MC; ++i) { zero8(pdy[i]); zero8(pdh[i]); zero8(py[i]); zero8(pb[i]); }
    };
    auto request = [&](int row, int end) {
        if (row >= end) return forget();
        if (pre) pr = a.pre_rstd[row];
        if (POST) pr2 = a.post_rstd[row];
        if (LN && a.pre == NORM_LAYER) pmu = a.pre_mean[row];
        if (SUM_B && a.post == NORM_LAYER) pmu2 = a.post_mean[row];
#pragma unroll
        for (int i = 0; i < MC; ++i) {
            if (col(i) >= H) continue;          // (these lanes keep the zeros they begin with)
            const size_t at = (size_t)row * H + col(i);
            if (a.dy) load_raw8((const T *)a.dy + at, pdy[i]);
            if (pre) { load_raw8((const T *)a.dh + at, pdh[i]); load_raw8((const T *)a.y + at, py[i]); }
            if (SUM_A) load_raw8((const T *)a.b + at, pb[i]);
        }
    };
#pragma unroll
    for (int i = 0; i < MC; ++i) {
        keep(w1, 0, i, a.pre_w);
        if constexpr (POST) keep(w2, 1, i, a.post_w);
        if constexpr (GATE) {
            zero8(gt[i]);
            if (a.gate == GATE_CHANNEL && inside(i)) gt[i] = load_plain8((const T *)a.gate_v + col(i));
        }
    }
    // two sums over the groups' rows, added in order, handed out in quads of columns, the same quads to the same thread every time
    auto flush = [&](const float (&p)[MC][8], const float (&q)[LN ? MC : 1][8], auto emit) {
        if constexpr (R == 1) {
#pragma unroll
            for (int i = 0; i < MC; ++i)
                if (col(i) < H) {
#pragma unroll
                    for (int j = 0; j < 8; j += 4) {
                        const int k = LN ? i : 0;
                        emit(col(i) + j, f32x4{p[i][j], p[i][j + 1], p[i][j + 2], p[i][j + 3]}, f32x4{q[k][j], q[k][j + 1], q[k][j + 2], q[k][j + 3]});
                    }
                }
        } else {
            __syncthreads();
#pragma unroll
            for (int i = 0; i < MC; ++i)
                if (col(i) < H) {
                    store8(&comb[0][grp][col(i)], p[i]);
                    if constexpr (LN) store8(&comb[1][grp][col(i)], q[i]);
                }
            __syncthreads();
            for (int c = threadIdx.x * 4; c < H; c += NT * 4) {
                f32x4 s[2] = {};
#pragma unroll
                for (int k = 0; k < (LN ? 2 : 1); ++k) {
                    s[k] = *reinterpret_cast<const f32x4 *>(&comb[k][0][c]);
#pragma unroll
                    for (int g = 1; g < R; ++g) s[k] += *reinterpret_cast<const f32x4 *>(&comb[k][g][c]);
                }
                emit(c, s[0], s[1]);
            }
        }
    };
    auto each_quad = [&](auto f) {                          // ... these quads
        if constexpr (R == 1) {
#pragma unroll
            for (int i = 0; i < MC; ++i)
                if (col(i) < H) { f(col(i)); f(col(i) + 4); }
        } else {
            for (int c = threadIdx.x * 4; c < H; c += NT * 4) f(c);
        }
    };
    auto quad = [](float *p) -> f32x4 & { return *reinterpret_cast<f32x4 *>(p); };
    // gradient of the gate from A and B: beta (w A + b B), or beta A
    auto gate_gradient = [&](int c, f32x4 sa, f32x4 sb) {
        if constexpr (POST) sa *= load4((const T *)a.post_w + c);
        if (SUM_B && a.post == NORM_LAYER) sa += sb * load4((const T *)a.post_b + c);
        return a.beta * sa;
    };
    request(r0 + grp, r1);
    for (int start = r0; start < r1;) {                     // start + grp is requested
        int end = r1, seg = 0;
        if constexpr (GATE) {
            if (by_segment) {
                seg = find_segment_wave(a.cu, a.S, start);
                end = min(r1, max(a.cu[seg + 1], start + 1));  // (goes on whatever the boundaries in memory are)
                if (start + grp >= end) forget();           // a row of the next segment: requested again in its turn
#pragma unroll
                for (int i = 0; i < MC; ++i)
                    if (col(i) < H) gt[i] = load_plain8((const T *)a.gate_v + (size_t)seg * H + col(i));
            }
        }
        for (int base = start; base < end; base += R) {
            const int row = base + grp;
            const bool valid = row < end;
            const float r = pr, mu = pmu, r2 = pr2, mu2 = pmu2;
            float d[MC][8], back[MC][8], hat[MC][8], bv[MC][8];
#pragma unroll
            for (int i = 0; i < MC; ++i) { unpack8(pdy[i], d[i]); unpack8(pdh[i], back[i]); unpack8(py[i], hat[i]); unpack8(pb[i], bv[i]); }
            const bool more = base + R < end;
            request(more ? row + R : end + grp, more ? end : r1);
            // no pre norm: r, dh and y are zero, and so is all of this
            float s0 = 0.f, s1 = 0.f, u0 = 0.f, u1 = 0.f;
#pragma unroll
            for (int i = 0; i < MC; ++i) {
                float g[8];
                unpack8(kept(w1, 0, i), g);
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    hat[i][j] = LN ? (hat[i][j] - mu) * r : hat[i][j] * r;
                    s_pre_w[i][j] += back[i][j] * hat[i][j];
                    if (LN) s_pre_b[i][j] += back[i][j];
                    back[i][j] *= g[j];
                    if (LN) s0 += back[i][j];
                    s1 += back[i][j] * hat[i][j];
                }
            }
            if constexpr (LN) row_sum(s0, s1);
            else row_sum(s1);
            s0 = LN && a.pre == NORM_LAYER ? s0 * inv_h : 0.f;
            s1 *= inv_h;
#pragma unroll
            for (int i = 0; i < MC; ++i) {
                float g[8], w[8], dx[8];
                if constexpr (GATE) unpack8(gt[i], g);
                if constexpr (POST) unpack8(kept(w2, 1, i), w);
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    d[i][j] += r * ((LN ? back[i][j] - s0 : back[i][j]) - hat[i][j] * s1);
                    dx[j] = alpha * d[i][j];
                    hat[i][j] = POST ? (LN ? (bv[i][j] - mu2) * r2 : bv[i][j] * r2) : bv[i][j];
                    if (SUM_A) sum_a[i][j] += d[i][j] * hat[i][j];
                    if (SUM_B) sum_b[i][j] += d[i][j];
                    back[i][j] = a.beta * d[i][j];
                    if (GATE) back[i][j] *= g[j];
                    if (POST) {
                        back[i][j] *= w[j];
                        if (LN) u0 += back[i][j];
                        u1 += back[i][j] * hat[i][j];
                    }
                }
                if (a.dx && valid && inside(i)) store8((T *)a.dx + (size_t)row * H + col(i), dx);
            }
            if constexpr (POST) {
                if constexpr (LN) row_sum(u0, u1);
                else row_sum(u1);
                u0 = LN && a.post == NORM_LAYER ? u0 * inv_h : 0.f;
                u1 *= inv_h;
#pragma unroll
                for (int i = 0; i < MC; ++i)
#pragma unroll
                    for (int j = 0; j < 8; ++j) back[i][j] = r2 * ((LN ? back[i][j] - u0 : back[i][j]) - hat[i][j] * u1);
            }
#pragma unroll
            for (int i = 0; i < MC; ++i)
                if (a.db && valid && inside(i)) store8((T *)a.db + (size_t)row * H + col(i), back[i]);
        }
        if constexpr (GATE) {
            if (by_segment) {
                const bool whole = a.cu[seg] >= r0 && a.cu[seg + 1] <= r1;
                const size_t out = (size_t)seg * H, slot = (2 * (size_t)block + (start != r0)) * H;
                flush(sum_a, sum_b, [&](int c, f32x4 sa, f32x4 sb) {
                    if (a.p_gate) {
                        const f32x4 g = gate_gradient(c, sa, sb);
                        if (!whole) quad(a.p_gate + slot + c) = g;
                        else if (a.grad_f32) quad((float *)a.d_gate + out + c) = a.accumulate ? quad((float *)a.d_gate + out + c) + g : g;
                        else store4((T *)a.d_gate + out + c, a.accumulate ? load4((const T *)a.d_gate + out + c) + g : g);
                    }
                    if constexpr (POST) {
                        const f32x4 g = a.beta * load4((const T *)a.gate_v + out + c);
                        quad(total_w + c) = start == r0 ? g * sa : quad(total_w + c) + g * sa;
                        if constexpr (SUM_B) quad(total_b + c) = start == r0 ? g * sb : quad(total_b + c) + g * sb;
                    }
                });
#pragma unroll
                for (int i = 0; i < MC; ++i)
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        sum_a[i][j] = 0.f;
                        if constexpr (LN) sum_b[i][j] = 0.f;
                    }
            }
        }
        start = end;
    }
    const size_t mine = (size_t)block * H;
    if (a.p_pre_w || a.p_pre_b)
        flush(s_pre_w, s_pre_b, [&](int c, f32x4 w, f32x4 b) {
            if (a.p_pre_w) quad(a.p_pre_w + mine + c) = w;
            if (LN && a.p_pre_b) quad(a.p_pre_b + mine + c) = b;
        });
    if (by_segment) {
        if constexpr (GATE && POST)
            each_quad([&](int c) {
                if (a.p_post_w) quad(a.p_post_w + mine + c) = quad(total_w + c);
                if constexpr (SUM_B) { if (a.p_post_b) quad(a.p_post_b + mine + c) = quad(total_b + c); }
            });
    } else if (SUM_A && (a.p_post_w || a.p_post_b || a.p_gate)) {
        flush(sum_a, sum_b, [&](int c, f32x4 sa, f32x4 sb) {
            f32x4 g = {a.beta, a.beta, a.beta, a.beta};
            if constexpr (GATE) g *= load4((const T *)a.gate_v + c);
            if (POST && a.p_post_w) quad(a.p_post_w + mine + c) = g * sa;
            if (SUM_B && a.p_post_b) quad(a.p_post_b + mine + c) = g * sb;
            if (GATE && a.p_gate) quad(a.p_gate + mine + c) = gate_gradient(c, sa, sb);
        });
    }
}

// What the backward kernel's workgroups leave behind, in one launch: the sums over their partial rows (reduce.h), then the gate gradients of the
// segments that several workgroups have rows of, then the zeros of the empty segments.
//
// A segment of the second kind begins in the range of one workgroup and goes on behind it: thread y of each of these workgroups looks at the end of
// workgroup y's range, the segments found are numbered in that order, and GATE_SHARES workgroups per 32 columns take them in turn.  Summed are
// slot 1 or 0 where the segment begins and slot 0 of each further workgroup, 32 rows at a time, in a fixed order.
constexpr int JOIN_BLOCKS = 256, GATE_SHARES = 8, GATE_EMPTY = 64;
struct GateSums {
    const float *part;
    void *out;                      // null: no segment gates
    const int *cu;
    int S, T, H, blocks, accumulate;
};
template <typename E>
__global__ __launch_bounds__(256) void join_sums_kernel(ReduceJobSet set, GateSums g) {
    __shared__ __attribute__((aligned(16))) float red[32][36];
    __shared__ int4 found[JOIN_BLOCKS];                     // segment, slot it begins in, first and last workgroup that goes on
    __shared__ int waves[4];
    const int units = set.units[8], tid = threadIdx.x;
    if ((int)blockIdx.x < units) return reduce_unit<E>(set, blockIdx.x, red, tid);
    const int columns = (g.H + 31) / 32, k = (int)blockIdx.x - units, c0 = k % columns * 32, share = k / columns;
    const int cl = tid & 7, rl = tid >> 3, c = c0 + cl * 4;
    E *out = (E *)g.out;
    if (share >= GATE_SHARES) {
        const int first = (share - GATE_SHARES) * GATE_EMPTY;
        for (int s = first + rl; s < min(first + GATE_EMPTY, g.S); s += 32)
            if (g.cu[s + 1] == g.cu[s] && c < g.H && !g.accumulate) {
#pragma unroll
                for (int j = 0; j < 4; ++j) Elem<E>::store(out + (size_t)s * g.H + c + j, 0.f);
            }
        return;
    }
    bool goes_on = false;
    int4 mine = {};
    if (tid < g.blocks) {
        const int r0 = join_row(g.T, g.blocks, tid), r1 = join_row(g.T, g.blocks, tid + 1);
        const int s = find_segment(g.cu, g.S, r1 - 1), b0 = g.cu[s], b1 = g.cu[s + 1];
        goes_on = b0 >= r0 && b1 > r1;
        const int q = g.T / g.blocks, longer = g.T % g.blocks, t = b1 - 1;      // the workgroup of row t
        mine = make_int4(s, 2 * tid + (b0 > r0), tid + 1, min(t < longer * (q + 1) ? t / (q + 1) : longer + (t - longer * (q + 1)) / q, g.blocks - 1));
    }
    const unsigned long long set_lanes = __ballot(goes_on);
    if ((tid & 63) == 0) waves[tid >> 6] = __popcll(set_lanes);
    __syncthreads();
    int before = 0, all = 0;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
        if (w < tid >> 6) before += waves[w];
        all += waves[w];
    }
    if (goes_on) found[before + __popcll(set_lanes & ((1ull << (tid & 63)) - 1))] = mine;
    __syncthreads();
    for (int i = share; i < all; i += GATE_SHARES) {
        const int4 f = found[i];
        f32x4 sum = {0.f, 0.f, 0.f, 0.f};
        if (c < g.H) {
            if (rl == 0) sum = *reinterpret_cast<const f32x4 *>(g.part + (size_t)f.y * g.H + c);
            for (int b = f.z + rl; b <= f.w; b += 32) sum += *reinterpret_cast<const f32x4 *>(g.part + (size_t)(2 * b) * g.H + c);
        }
        __syncthreads();
        *reinterpret_cast<f32x4 *>(&red[rl][cl * 4]) = sum;
        __syncthreads();
        if (tid < 32 && c0 + tid < g.H) {
            float t = 0.f;
#pragma unroll
            for (int r = 0; r < 32; ++r) t += red[r][tid];
            E *o = out + (size_t)f.x * g.H + c0 + tid;
            if (g.accumulate) t += Elem<E>::load(o);
            Elem<E>::store(o, t);
        }
    }
}

template <typename F> auto with(bool v, F f) { return v ? f(std::true_type{}) : f(std::false_type{}); }

template <typename T, int G, int MC, int NT, bool LN>
hipError_t launch_fwd(const JoinArgs &a, hipStream_t st) {
    return with(a.gate != GATE_NONE, [&](auto GATE) {
        return with(a.post != NORM_NONE, [&](auto POST) {
            static std::atomic<int> resident{0};
            auto kern = join_fwd_kernel<T, G, MC, NT, LN, decltype(GATE)::value, decltype(POST)::value>;
            int grid = 0;
            const hipError_t e = resident_workgroups(resident, kern, grid, NT);
            if (e != hipSuccess) return e;
            const int all = ceil_div(a.T, NT / G);
            kern<<<all < grid ? all : grid, NT, 0, st>>>(a);
            return hipGetLastError();
        });
    });
}

template <typename T, int G, int MC, int NT>
hipError_t launch_bwd(const JoinArgs &a, hipStream_t st) {
    const int blocks = join_bwd_blocks(a.T, a.H);
    return with(a.post == NORM_LAYER || a.pre == NORM_LAYER, [&](auto LN) {
        return with(a.gate != GATE_NONE, [&](auto GATE) {
            return with(a.post != NORM_NONE, [&](auto POST) {
                join_bwd_kernel<T, G, MC, NT, decltype(LN)::value, decltype(GATE)::value, decltype(POST)::value><<<blocks, NT, 0, st>>>(a);
                return hipGetLastError();
            });
        });
    });
}

// By width: threads a row, chunks a thread, threads a workgroup.  Few idle lanes in a row, and few enough registers for two workgroups per compute unit or
// more, so that one's sums go on beside another's loads.  9000 bf16 rows forward, two RMSNorms / two LayerNorms and a gate, us, the row's class against the
// next best: 1024 (128, 1) 15.0 / 18.3, (64, 2) 15.1 / 21.7; 1280 192 threads a workgroup 21.2 / 23.0, 384 17.7 / 30.8, so the latter where there is no mean;
// 4096 (512, 1) 60.3 / 63.6, (256, 2) 61.6 / 66.3; the same class at 2560 and 3584, where 192 and 64 of its threads have no columns, 37.7 / 45.9 and 52.9 / 56.0
// (bytes at 5 TB/s: 36.9 and 51.6; no class between was tried); 5120 (640, 1) 79.4 / 96.4, (384, 2) 78.9 / 89.7 (fp32 151 / 154, 155 / 165); 8192 (512, 2) 129 / 147, (1024, 1) 122 / 155, so the latter where there is no mean.
template <typename T>
hipError_t fwd_by_width(const JoinArgs &a, hipStream_t st) {
    const bool ln = a.post == NORM_LAYER || a.pre == NORM_LAYER;
#define L(G, MC, NT) (ln ? launch_fwd<T, G, MC, NT, true>(a, st) : launch_fwd<T, G, MC, NT, false>(a, st))
    if (a.H <= 64 * 8) return L(64, 1, 256);
    if (a.H <= 128 * 8) return L(128, 1, 256);
    if (a.H <= 192 * 8) return ln ? launch_fwd<T, 192, 1, 192, true>(a, st) : launch_fwd<T, 192, 1, 384, false>(a, st);
    if (a.H <= 256 * 8) return ln ? launch_fwd<T, 256, 1, 256, true>(a, st) : launch_fwd<T, 256, 1, 512, false>(a, st);
    if (a.H <= 512 * 8) return L(512, 1, 512);
    if (a.H <= 640 * 8) {
        if (ln && sizeof(T) == 2) return launch_fwd<T, 384, 2, 384, true>(a, st);
        return L(640, 1, 640);
    }
    return ln ? launch_fwd<T, 512, 2, 512, true>(a, st) : launch_fwd<T, 1024, 1, 1024, false>(a, st);
#undef L
}
// Backward, where a workgroup has the compute unit to itself: as many threads as have the registers.  9000 bf16 rows, two RMSNorms / two LayerNorms and a gate
// per segment, us: 1024 (128, 1) 26.8 / 34.0, (64, 2) 27.2 / 35.3 (in fp32 55 / 62, 55 / 79: it spills); 1280 768 threads a workgroup 31.5 / 39.2, 576 31.8 / 40.9; 4096
// (512, 1) 98.1 / 110, (256, 2) 97.0 / 110 (fp32 186 / 198, 188 / 214); the same class at 2560 and 3584 63.5 / 72.6 and 84.6 / 93.9 (bytes 55.3 and 77.4; no class
// between was tried); 5120 (640, 1) 118 / 130, (384, 2) 119 / 134; 8192 (512, 2) 192 / 211, (1024, 1) 192 / 622.
template <typename T>
hipError_t bwd_by_width(const JoinArgs &a, hipStream_t st) {
    if (a.H <= 64 * 8) return launch_bwd<T, 64, 1, 512>(a, st);
    if (a.H <= 128 * 8) return launch_bwd<T, 128, 1, 768>(a, st);
    if (a.H <= 192 * 8) return launch_bwd<T, 192, 1, 768>(a, st);
    if (a.H <= 256 * 8) return launch_bwd<T, 256, 1, 768>(a, st);
    if (a.H <= 512 * 8) return launch_bwd<T, 512, 1, 512>(a, st);
    if (a.H <= 640 * 8) return launch_bwd<T, 640, 1, 640>(a, st);
    return launch_bwd<T, 512, 2, 512>(a, st);
}

}  // namespace

hipError_t join_fwd(int dtype, const JoinArgs &a, hipStream_t st) {
    if (a.T == 0) return hipSuccess;
    return dtype == DT_F32 ? fwd_by_width<float>(a, st) : fwd_by_width<bf16_t>(a, st);
}

// as many as there are rows at a time, at most one per compute unit
int join_bwd_blocks(int T, int H) {
    const int at_once = H <= 64 * 8 ? 8 : H <= 128 * 8 ? 6 : H <= 192 * 8 ? 4 : H <= 256 * 8 ? 3 : 1;
    return std::min(ceil_div(T, at_once), JOIN_BLOCKS);
}

hipError_t join_bwd(int dtype, const JoinArgs &a, hipStream_t st) {
    const int blocks = join_bwd_blocks(a.T, a.H);
    if (a.T > 0) {
        const hipError_t e = dtype == DT_F32 ? bwd_by_width<float>(a, st) : bwd_by_width<bf16_t>(a, st);
        if (e != hipSuccess) return e;
    }
    const bool by_segment = a.gate == GATE_SEGMENT && a.d_gate && a.S > 0;
    const ReduceJob jobs[5] = {{a.p_post_w, a.d_post_w, blocks, a.H}, {a.p_post_b, a.d_post_b, blocks, a.H}, {a.p_pre_w, a.d_pre_w, blocks, a.H},
                               {a.p_pre_b, a.d_pre_b, blocks, a.H}, {a.gate == GATE_CHANNEL ? a.p_gate : nullptr, a.d_gate, blocks, a.H}};
    ReduceJobSet set;
    reduce_job_set(jobs, 5, a.accumulate, set);
    const GateSums g = {a.p_gate, by_segment ? a.d_gate : nullptr, a.cu, a.S, a.T, a.H, blocks, a.accumulate};
    const int grid = set.units[8] + (by_segment ? ceil_div(a.H, 32) * (GATE_SHARES + ceil_div(a.S, GATE_EMPTY)) : 0);
    if (grid == 0) return hipSuccess;
    if (a.grad_f32) join_sums_kernel<float><<<grid, 256, 0, st>>>(set, g);
    else join_sums_kernel<bf16_t><<<grid, 256, 0, st>>>(set, g);
    return hipGetLastError();
}

}  // namespace mmt
