// The join of a block's branch with the residual stream: norm behind the block, gate, scales, norm in front of the next.
//     n = norm_post(b);  y = alpha x + beta gate n;  h = norm_pre(y)
//
// Memory-bound: forward reads x and b and writes y and h, backward reads dy, dh, y and b and writes dx and db, each once; a row stays in
// registers from its first use to its last.  A row is worked on by a group of G threads with MC chunks of 8 columns each -- a wavefront
// up to 1024 columns, where sums need no barrier -- and a workgroup of NT threads walks over a contiguous range of rows, NT / G at a
// time, the next ones requested before the present ones are reduced.  Gains, biases and gates stay in registers; so do backward's
// sums over tokens, which leave the workgroup as one partial row.
#include "ops.h"
#include "vec8.h"
#include "resident.h"
#include <type_traits>

namespace mmt {
namespace {

// first row of workgroup b of `blocks`
__device__ __forceinline__ int join_row(int T, int blocks, int b) { return (int)((long)T * b / blocks); }

// Sums over the G threads of a row.  red: two buffers, used in turn, so that one barrier per sum is enough (a thread that writes a buffer
// again has passed the barrier behind its last reading).  All threads of the workgroup call it together.
template <int G, int NT> struct RowSum {
    float (*red)[NT / 64][2];
    int turn = 0;
    __device__ __forceinline__ void operator()(float &a, float &b) {
        a = wave_sum(a); b = wave_sum(b);
        if constexpr (G == 64) return;
        const int wave = threadIdx.x >> 6, first = (threadIdx.x / G) * (G / 64);
        if ((threadIdx.x & 63) == 0) { red[turn][wave][0] = a; red[turn][wave][1] = b; }
        __syncthreads();
        a = b = 0.f;
#pragma unroll
        for (int i = 0; i < G / 64; ++i) { a += red[turn][first + i][0]; b += red[turn][first + i][1]; }
        turn ^= 1;
    }
    __device__ __forceinline__ float operator()(float a) {
        a = wave_sum(a);
        if constexpr (G == 64) return a;
        const int wave = threadIdx.x >> 6, first = (threadIdx.x / G) * (G / 64);
        if ((threadIdx.x & 63) == 0) red[turn][wave][0] = a;
        __syncthreads();
        a = 0.f;
#pragma unroll
        for (int i = 0; i < G / 64; ++i) a += red[turn][first + i][0];
        turn ^= 1;
        return a;
    }
};

template <typename T> __device__ __forceinline__ void zero8(Raw8<T> &r) { __builtin_memset(&r, 0, sizeof(r)); }

// LN: one of the norms is a LayerNorm (gains only otherwise)
template <typename T, int G, int MC, int NT, bool LN>
__global__ __launch_bounds__(NT) void join_fwd_kernel(JoinArgs a) {
    constexpr int R = NT / G;
    __shared__ float red_[2][NT / 64][2];
    RowSum<G, NT> row_sum{red_};
    const int lane = threadIdx.x % G, grp = threadIdx.x / G, H = a.H;
    const int r0 = join_row(a.T, gridDim.x, blockIdx.x), r1 = join_row(a.T, gridDim.x, blockIdx.x + 1);
    const float inv_h = 1.f / H;
    auto col = [&](int i) { return (lane + i * G) * 8; };
    Raw8<T> nx[MC], nb[MC], w2[MC], w1[MC], gt[MC], b2[LN ? MC : 1], b1[LN ? MC : 1];
    auto request = [&](int row) {
#pragma unroll
        for (int i = 0; i < MC; ++i) {
            zero8(nx[i]); zero8(nb[i]);
            if (col(i) >= H || row >= r1) continue;
            const size_t at = (size_t)row * H + col(i);
            load_raw8((const T *)a.x + at, nx[i]);
            if (a.b) load_raw8((const T *)a.b + at, nb[i]);
        }
    };
    request(r0 + grp);
#pragma unroll
    for (int i = 0; i < MC; ++i) {
        if (col(i) >= H) continue;
        if (a.post != NORM_NONE) w2[i] = load_plain8((const T *)a.post_w + col(i));
        if (a.pre != NORM_NONE) w1[i] = load_plain8((const T *)a.pre_w + col(i));
        if (LN && a.post == NORM_LAYER) b2[i] = load_plain8((const T *)a.post_b + col(i));
        if (LN && a.pre == NORM_LAYER) b1[i] = load_plain8((const T *)a.pre_b + col(i));
        if (a.gate == GATE_CHANNEL) gt[i] = load_plain8((const T *)a.gate_v + col(i));
    }
    int seg_end = 0;
    // v <- normalised v, gain and bias applied
    auto norm = [&](float (&v)[MC][8], int kind, float eps, const Raw8<T> (&w)[MC], const Raw8<T> *bias, float &mu, float &r) {
        mu = 0.f;
        if (LN && kind == NORM_LAYER) {
            float s = 0.f;
#pragma unroll
            for (int i = 0; i < MC; ++i)
#pragma unroll
                for (int j = 0; j < 8; ++j) s += v[i][j];
            mu = row_sum(s) * inv_h;
        }
        float q = 0.f;
#pragma unroll
        for (int i = 0; i < MC; ++i)
            if (col(i) < H) {
#pragma unroll
                for (int j = 0; j < 8; ++j) q += (v[i][j] - mu) * (v[i][j] - mu);
            }
        r = 1.f / sqrtf(row_sum(q) * inv_h + eps);
#pragma unroll
        for (int i = 0; i < MC; ++i) {
            float g[8], o[8];
            unpack8(w[i], g);
            if (LN && kind == NORM_LAYER) unpack8(bias[i], o);
#pragma unroll
            for (int j = 0; j < 8; ++j) v[i][j] = (v[i][j] - mu) * r * g[j] + (LN && kind == NORM_LAYER ? o[j] : 0.f);
        }
    };
    for (int base = r0; base < r1; base += R) {
        const int row = base + grp;
        const bool valid = row < r1;
        float xv[MC][8], v[MC][8], mu, r;
#pragma unroll
        for (int i = 0; i < MC; ++i) { unpack8(nx[i], xv[i]); unpack8(nb[i], v[i]); }
        request(row + R);
        if (a.b) {
            if (a.gate == GATE_SEGMENT && valid && row >= seg_end) {
                const int seg = find_segment(a.cu, a.S, row);
                seg_end = a.cu[seg + 1];
#pragma unroll
                for (int i = 0; i < MC; ++i)
                    if (col(i) < H) gt[i] = load_plain8((const T *)a.gate_v + (size_t)seg * H + col(i));
            }
            if (a.post != NORM_NONE) {
                norm(v, a.post, a.post_eps, w2, b2, mu, r);
                if (lane == 0 && valid) {
                    if (a.post_rstd) a.post_rstd[row] = r;
                    if (LN && a.post == NORM_LAYER && a.post_mean) a.post_mean[row] = mu;
                }
            }
#pragma unroll
            for (int i = 0; i < MC; ++i) {
                float g[8];
                if (a.gate != GATE_NONE) unpack8(gt[i], g);
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    v[i][j] = col(i) < H ? a.alpha * xv[i][j] + a.beta * (a.gate != GATE_NONE ? g[j] : 1.f) * v[i][j] : 0.f;
                if (valid && col(i) < H) store8((T *)a.y + (size_t)row * H + col(i), v[i]);
            }
        } else {
#pragma unroll
            for (int i = 0; i < MC; ++i)
#pragma unroll
                for (int j = 0; j < 8; ++j) v[i][j] = xv[i][j];
        }
        if (a.pre == NORM_NONE) continue;
        norm(v, a.pre, a.pre_eps, w1, b1, mu, r);
        if (lane == 0 && valid) {
            if (a.pre_rstd) a.pre_rstd[row] = r;
            if (LN && a.pre == NORM_LAYER && a.pre_mean) a.pre_mean[row] = mu;
        }
#pragma unroll
        for (int i = 0; i < MC; ++i)
            if (valid && col(i) < H) store8((T *)a.h + (size_t)row * H + col(i), v[i]);
    }
}

// With hat = (v - mean) r and back = d_out w, a norm's input gradient is r (back - mean(back) [LAYER] - hat mean(back hat)); gain and bias
// get sum d_out hat and sum d_out.  Gradient of y: d = dy + the pre norm's; then dx = alpha d, the branch gets beta gate d through the
// post norm, and the gate sum beta n d.
//
// By segment, a workgroup's gate sums go out at the end of each segment's rows: as the gradient where it has all of them, else into its
// slot 0 if its range begins inside the segment or with it, and into slot 1 otherwise (then the range ends in it).
template <typename T, int G, int MC, int NT, bool LN, bool GATE>
__global__ __launch_bounds__(NT) void join_bwd_kernel(JoinArgs a) {
    constexpr int R = NT / G, W = G * MC * 8;
    __shared__ float red_[2][NT / 64][2];
    __shared__ __attribute__((aligned(16))) float comb[R > 1 ? R : 1][R > 1 ? W : 4];
    RowSum<G, NT> row_sum{red_};
    const int lane = threadIdx.x % G, grp = threadIdx.x / G, H = a.H, block = blockIdx.x;
    const int r0 = join_row(a.T, gridDim.x, block), r1 = join_row(a.T, gridDim.x, block + 1);
    const float inv_h = 1.f / H;
    const bool pre = a.pre != NORM_NONE, post = a.post != NORM_NONE, by_segment = GATE && a.gate == GATE_SEGMENT;
    auto col = [&](int i) { return (lane + i * G) * 8; };
    Raw8<T> pdy[MC], pdh[MC], py[MC], pb[MC], w1[MC], w2[MC], gt[GATE ? MC : 1], b2[LN && GATE ? MC : 1];
    float s_pre_w[MC][8] = {}, s_post_w[MC][8] = {}, s_pre_b[LN ? MC : 1][8] = {}, s_post_b[LN ? MC : 1][8] = {}, s_gate[GATE ? MC : 1][8] = {};
    float pr = 0.f, pmu = 0.f, pr2 = 0.f, pmu2 = 0.f;
    auto request = [&](int row, int end) {
        const bool in = row < end;
        pr = pmu = pr2 = pmu2 = 0.f;
        if (in) {
            if (pre) pr = a.pre_rstd[row];
            if (post) pr2 = a.post_rstd[row];
            if (LN && a.pre == NORM_LAYER) pmu = a.pre_mean[row];
            if (LN && a.post == NORM_LAYER) pmu2 = a.post_mean[row];
        }
#pragma unroll
        for (int i = 0; i < MC; ++i) {
            zero8(pdy[i]); zero8(pdh[i]); zero8(py[i]); zero8(pb[i]);
            if (!in || col(i) >= H) continue;
            const size_t at = (size_t)row * H + col(i);
            if (a.dy) load_raw8((const T *)a.dy + at, pdy[i]);
            if (pre) { load_raw8((const T *)a.dh + at, pdh[i]); load_raw8((const T *)a.y + at, py[i]); }
            if (post || (GATE && a.b)) load_raw8((const T *)a.b + at, pb[i]);
        }
    };
#pragma unroll
    for (int i = 0; i < MC; ++i) {
        if (col(i) >= H) continue;
        if (pre) w1[i] = load_plain8((const T *)a.pre_w + col(i));
        if (post) w2[i] = load_plain8((const T *)a.post_w + col(i));
        if (LN && GATE && a.post == NORM_LAYER) b2[i] = load_plain8((const T *)a.post_b + col(i));
        if (GATE && a.gate == GATE_CHANNEL) gt[i] = load_plain8((const T *)a.gate_v + col(i));
    }
    // the sums of the groups, added in order, handed out in quads of columns
    auto flush = [&](const float (&v)[MC][8], auto emit) {
        if constexpr (R == 1) {
#pragma unroll
            for (int i = 0; i < MC; ++i)
                if (col(i) < H) {
                    emit(col(i), f32x4{v[i][0], v[i][1], v[i][2], v[i][3]});
                    emit(col(i) + 4, f32x4{v[i][4], v[i][5], v[i][6], v[i][7]});
                }
        } else {
            __syncthreads();
#pragma unroll
            for (int i = 0; i < MC; ++i)
                if (col(i) < H) store8(&comb[grp][col(i)], v[i]);
            __syncthreads();
            for (int c = threadIdx.x * 4; c < H; c += NT * 4) {
                f32x4 s = *reinterpret_cast<const f32x4 *>(&comb[0][c]);
#pragma unroll
                for (int g = 1; g < R; ++g) s += *reinterpret_cast<const f32x4 *>(&comb[g][c]);
                emit(c, s);
            }
        }
    };
    auto to_part = [&](float *part, size_t row) {
        return [=](int c, f32x4 s) { *reinterpret_cast<f32x4 *>(part + row * H + c) = s; };
    };
    for (int start = r0; start < r1;) {
        int end = r1, seg = 0;
        if constexpr (GATE) {
            if (by_segment) {
                seg = find_segment(a.cu, a.S, start);
                end = min(r1, a.cu[seg + 1]);
#pragma unroll
                for (int i = 0; i < MC; ++i)
                    if (col(i) < H) gt[i] = load_plain8((const T *)a.gate_v + (size_t)seg * H + col(i));
            }
        }
        request(start + grp, end);
        for (int base = start; base < end; base += R) {
            const int row = base + grp;
            const bool valid = row < end;
            const float r = pr, mu = pmu, r2 = pr2, mu2 = pmu2;
            float d[MC][8], back[MC][8], hat[MC][8], bv[MC][8];
#pragma unroll
            for (int i = 0; i < MC; ++i) { unpack8(pdy[i], d[i]); unpack8(pdh[i], back[i]); unpack8(py[i], hat[i]); unpack8(pb[i], bv[i]); }
            request(row + R, end);
            if (pre) {
                float s0 = 0.f, s1 = 0.f;
#pragma unroll
                for (int i = 0; i < MC; ++i) {
                    if (col(i) >= H) continue;
                    float g[8];
                    unpack8(w1[i], g);
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        hat[i][j] = (hat[i][j] - mu) * r;
                        s_pre_w[i][j] += back[i][j] * hat[i][j];
                        if (LN) s_pre_b[i][j] += back[i][j];
                        back[i][j] *= g[j];
                        s0 += back[i][j];
                        s1 += back[i][j] * hat[i][j];
                    }
                }
                row_sum(s0, s1);
                s0 = LN && a.pre == NORM_LAYER ? s0 * inv_h : 0.f;
                s1 *= inv_h;
#pragma unroll
                for (int i = 0; i < MC; ++i)
#pragma unroll
                    for (int j = 0; j < 8; ++j) d[i][j] += r * (back[i][j] - s0 - hat[i][j] * s1);
            }
            if (!a.b) {
#pragma unroll
                for (int i = 0; i < MC; ++i)
                    if (a.dx && valid && col(i) < H) store8((T *)a.dx + (size_t)row * H + col(i), d[i]);
                continue;
            }
            float u0 = 0.f, u1 = 0.f;
#pragma unroll
            for (int i = 0; i < MC; ++i) {
                if (col(i) >= H) continue;
                float g[8], w[8], o[8], dx[8];
                if constexpr (GATE) unpack8(gt[i], g);
                if (post) unpack8(w2[i], w);
                if constexpr (LN && GATE) { if (a.post == NORM_LAYER) unpack8(b2[i], o); }
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    dx[j] = a.alpha * d[i][j];
                    const float dn = a.beta * d[i][j];
                    float n = bv[i][j];
                    back[i][j] = GATE ? dn * g[j] : dn;
                    if (post) {
                        n = hat[i][j] = (n - mu2) * r2;
                        s_post_w[i][j] += back[i][j] * n;
                        if (LN) s_post_b[i][j] += back[i][j];
                        back[i][j] *= w[j];
                        u0 += back[i][j];
                        u1 += back[i][j] * n;
                        if (GATE) n = n * w[j] + (LN && a.post == NORM_LAYER ? o[j] : 0.f);
                    }
                    if (GATE) s_gate[i][j] += dn * n;
                }
                if (a.dx && valid) store8((T *)a.dx + (size_t)row * H + col(i), dx);
            }
            if (post) {
                row_sum(u0, u1);
                u0 = LN && a.post == NORM_LAYER ? u0 * inv_h : 0.f;
                u1 *= inv_h;
#pragma unroll
                for (int i = 0; i < MC; ++i)
#pragma unroll
                    for (int j = 0; j < 8; ++j) back[i][j] = r2 * (back[i][j] - u0 - hat[i][j] * u1);
            }
#pragma unroll
            for (int i = 0; i < MC; ++i)
                if (a.db && valid && col(i) < H) store8((T *)a.db + (size_t)row * H + col(i), back[i]);
        }
        if constexpr (GATE) {
            if (by_segment && a.p_gate) {
                if (a.cu[seg] >= r0 && a.cu[seg + 1] <= r1) {
                    flush(s_gate, [&](int c, f32x4 s) {
                        const size_t at = (size_t)seg * H + c;
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            if (a.grad_f32) ((float *)a.d_gate)[at + j] = s[j] + (a.accumulate ? ((float *)a.d_gate)[at + j] : 0.f);
                            else Elem<T>::store((T *)a.d_gate + at + j, s[j] + (a.accumulate ? Elem<T>::load((T *)a.d_gate + at + j) : 0.f));
                        }
                    });
                } else {
                    flush(s_gate, to_part(a.p_gate, 2 * (size_t)block + (start != r0)));
                }
#pragma unroll
                for (int i = 0; i < MC; ++i)
#pragma unroll
                    for (int j = 0; j < 8; ++j) s_gate[i][j] = 0.f;
            }
        }
        start = end;
    }
    if (a.p_pre_w) flush(s_pre_w, to_part(a.p_pre_w, block));
    if (a.p_post_w) flush(s_post_w, to_part(a.p_post_w, block));
    if constexpr (LN) {
        if (a.p_pre_b) flush(s_pre_b, to_part(a.p_pre_b, block));
        if (a.p_post_b) flush(s_post_b, to_part(a.p_post_b, block));
    }
    if constexpr (GATE) {
        if (a.p_gate && !by_segment) flush(s_gate, to_part(a.p_gate, block));
    }
}

// The gradient of a segment's gate where several workgroups have rows of the segment: their slots, in order.  No row: zero.
template <typename G>
__global__ __launch_bounds__(256) void gate_segments_kernel(const float *part, const int *cu, int T, int H, int blocks, G *out, bool accumulate) {
    const int s = blockIdx.y, c = blockIdx.x * 256 + threadIdx.x, b0 = cu[s], b1 = cu[s + 1];
    if (c >= H) return;
    float sum = 0.f;
    if (b1 > b0) {
        // the workgroup of row t: the last one whose first row is t or before
        auto owner = [&](int t) {
            int b = (int)((long)t * blocks / T);
            while (b + 1 < blocks && join_row(T, blocks, b + 1) <= t) ++b;
            while (join_row(T, blocks, b) > t) --b;
            return b;
        };
        const int first = owner(b0), last = owner(b1 - 1);
        if (first == last) return;
        for (int b = first; b <= last; ++b) sum += part[(size_t)(2 * b + (join_row(T, blocks, b) < b0)) * H + c];
    }
    const size_t at = (size_t)s * H + c;
    if (accumulate) sum += Elem<G>::load(out + at);
    Elem<G>::store(out + at, sum);
}

template <typename T, int G, int MC, int NT, bool LN>
hipError_t launch_fwd(const JoinArgs &a, hipStream_t st) {
    static std::atomic<int> resident{0};
    auto kern = join_fwd_kernel<T, G, MC, NT, LN>;
    int grid = 0;
    hipError_t e = resident_workgroups(resident, kern, grid, NT);
    if (e != hipSuccess) return e;
    const int all = ceil_div(a.T, NT / G);
    kern<<<all < grid ? all : grid, NT, 0, st>>>(a);
    return hipGetLastError();
}

template <typename T, int G, int MC, int NT>
hipError_t launch_bwd(const JoinArgs &a, hipStream_t st) {
    const bool ln = a.post == NORM_LAYER || a.pre == NORM_LAYER, gate = a.gate != GATE_NONE;
    const int blocks = join_bwd_blocks(a.T, a.H);
    if (ln && gate) join_bwd_kernel<T, G, MC, NT, true, true><<<blocks, NT, 0, st>>>(a);
    else if (ln) join_bwd_kernel<T, G, MC, NT, true, false><<<blocks, NT, 0, st>>>(a);
    else if (gate) join_bwd_kernel<T, G, MC, NT, false, true><<<blocks, NT, 0, st>>>(a);
    else join_bwd_kernel<T, G, MC, NT, false, false><<<blocks, NT, 0, st>>>(a);
    return hipGetLastError();
}

// by width: (threads a row, chunks a thread, threads a workgroup)
constexpr int BWD_ROWS_WAVE = 4, BWD_ROWS_WIDE = 2;
template <typename T>
hipError_t fwd_by_width(const JoinArgs &a, hipStream_t st) {
    const bool ln = a.post == NORM_LAYER || a.pre == NORM_LAYER;
#define L(G, MC, NT) return ln ? launch_fwd<T, G, MC, NT, true>(a, st) : launch_fwd<T, G, MC, NT, false>(a, st)
    if (a.H <= 512) L(64, 1, 256);
    if (a.H <= 1024) L(64, 2, 256);
    if (a.H <= 2048) L(256, 1, 256);
    if (a.H <= 4096) L(256, 2, 256);
    L(512, 2, 512);
#undef L
}
template <typename T>
hipError_t bwd_by_width(const JoinArgs &a, hipStream_t st) {
    if (a.H <= 512) return launch_bwd<T, 64, 1, 64 * BWD_ROWS_WAVE>(a, st);
    if (a.H <= 1024) return launch_bwd<T, 64, 2, 64 * BWD_ROWS_WAVE>(a, st);
    if (a.H <= 2048) return launch_bwd<T, 256, 1, 256 * BWD_ROWS_WIDE>(a, st);
    if (a.H <= 4096) return launch_bwd<T, 256, 2, 256 * BWD_ROWS_WIDE>(a, st);
    return launch_bwd<T, 512, 2, 512>(a, st);
}

}  // namespace

hipError_t join_fwd(int dtype, const JoinArgs &a, hipStream_t st) {
    if (a.T == 0) return hipSuccess;
    return dtype == DT_F32 ? fwd_by_width<float>(a, st) : fwd_by_width<bf16_t>(a, st);
}

int join_bwd_blocks(int T, int H) {
    const int all = H <= 1024 ? ceil_div(T, BWD_ROWS_WAVE) : H <= 4096 ? ceil_div(T, BWD_ROWS_WIDE) : T;
    return all < 512 ? all : 512;
}

hipError_t join_bwd(int dtype, const JoinArgs &a, hipStream_t st) {
    const int blocks = join_bwd_blocks(a.T, a.H);
    if (a.T > 0) {
        const hipError_t e = dtype == DT_F32 ? bwd_by_width<float>(a, st) : bwd_by_width<bf16_t>(a, st);
        if (e != hipSuccess) return e;
    }
    if (a.gate != GATE_SEGMENT || !a.d_gate || a.S == 0) return hipSuccess;
    for (int s = 0; s < a.S; s += 65535) {          // a grid's second dimension ends there
        const dim3 grid(ceil_div(a.H, 256), a.S - s < 65535 ? a.S - s : 65535);
        const size_t at = (size_t)s * a.H;
        if (a.grad_f32) gate_segments_kernel<float><<<grid, 256, 0, st>>>(a.p_gate, a.cu + s, a.T, a.H, blocks, (float *)a.d_gate + at, a.accumulate);
        else gate_segments_kernel<bf16_t><<<grid, 256, 0, st>>>(a.p_gate, a.cu + s, a.T, a.H, blocks, (bf16_t *)a.d_gate + at, a.accumulate);
    }
    return hipGetLastError();
}

}  // namespace mmt
