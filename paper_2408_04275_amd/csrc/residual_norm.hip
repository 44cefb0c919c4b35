// The join of a block's branch with the residual stream: norm behind the block, gate, scales, norm in front of the next.
#include "ops.h"

namespace mmt {
namespace {

// first row of workgroup b of `blocks`
__device__ __forceinline__ int join_row(int T, int blocks, int b) { return (int)((long)T * b / blocks); }

// mean and 1 / deviation of a row, whose elements v(c) gives
template <typename V>
__device__ __forceinline__ void row_statistics(int H, int kind, float eps, float *red, V v, float &mu, float &r) {
    mu = 0.f;
    if (kind == NORM_LAYER) {
        float s = 0.f;
        for (int c = threadIdx.x; c < H; c += 256) s += v(c);
        mu = block_sum<4>(s, red) / H;
    }
    float q = 0.f;
    for (int c = threadIdx.x; c < H; c += 256) q += (v(c) - mu) * (v(c) - mu);
    r = 1.f / sqrtf(block_sum<4>(q, red) / H + eps);
}

template <typename T>
__global__ __launch_bounds__(256) void join_fwd_kernel(JoinArgs a) {
    __shared__ float red[4];
    __shared__ float row[8192];
    const int t = blockIdx.x;
    const T *x = (const T *)a.x + (size_t)t * a.H, *b = a.b ? (const T *)a.b + (size_t)t * a.H : nullptr;
    const T *gate = (const T *)a.gate_v;
    if (a.gate == GATE_SEGMENT) gate += (size_t)find_segment(a.cu, a.S, t) * a.H;
    float mu, r;
    if (b) {
        if (a.post != NORM_NONE) {
            row_statistics(a.H, a.post, a.post_eps, red, [&](int c) { return Elem<T>::load(b + c); }, mu, r);
            if (threadIdx.x == 0) {
                if (a.post_rstd) a.post_rstd[t] = r;
                if (a.post == NORM_LAYER && a.post_mean) a.post_mean[t] = mu;
            }
        }
        for (int c = threadIdx.x; c < a.H; c += 256) {
            float n = Elem<T>::load(b + c);
            if (a.post != NORM_NONE) n = (n - mu) * r * Elem<T>::load((const T *)a.post_w + c);
            if (a.post == NORM_LAYER) n += Elem<T>::load((const T *)a.post_b + c);
            if (a.gate != GATE_NONE) n *= Elem<T>::load(gate + c);
            row[c] = a.alpha * Elem<T>::load(x + c) + a.beta * n;
            Elem<T>::store((T *)a.y + (size_t)t * a.H + c, row[c]);
        }
    } else {
        for (int c = threadIdx.x; c < a.H; c += 256) row[c] = Elem<T>::load(x + c);
    }
    if (a.pre == NORM_NONE) return;
    row_statistics(a.H, a.pre, a.pre_eps, red, [&](int c) { return row[c]; }, mu, r);
    if (threadIdx.x == 0) {
        if (a.pre_rstd) a.pre_rstd[t] = r;
        if (a.pre == NORM_LAYER && a.pre_mean) a.pre_mean[t] = mu;
    }
    for (int c = threadIdx.x; c < a.H; c += 256) {
        float n = (row[c] - mu) * r * Elem<T>::load((const T *)a.pre_w + c);
        if (a.pre == NORM_LAYER) n += Elem<T>::load((const T *)a.pre_b + c);
        Elem<T>::store((T *)a.h + (size_t)t * a.H + c, n);
    }
}

// A workgroup's gate sums of segment s: written as the gradient where it has all of the segment's rows, else into its slot 0 if the
// segment is its first and into slot 1 otherwise (then it is its last).
template <typename T>
__global__ __launch_bounds__(256) void join_bwd_kernel(JoinArgs a) {
    __shared__ float red[4];
    __shared__ float total[8192];                   // gradient of y
    const int blocks = gridDim.x, r0 = join_row(a.T, blocks, blockIdx.x), r1 = join_row(a.T, blocks, blockIdx.x + 1);
    const T *gate = (const T *)a.gate_v;
    int seg = -1, seg_end = 0, first_seg = -1;
    const bool by_segment = a.gate == GATE_SEGMENT;
    const size_t base = (size_t)blockIdx.x * a.H;
    for (int c = threadIdx.x; c < a.H; c += 256) {
        if (a.p_post_w) a.p_post_w[base + c] = 0.f;
        if (a.p_post_b) a.p_post_b[base + c] = 0.f;
        if (a.p_pre_w) a.p_pre_w[base + c] = 0.f;
        if (a.p_pre_b) a.p_pre_b[base + c] = 0.f;
        if (a.p_gate && !by_segment) a.p_gate[base + c] = 0.f;
    }
    float *gate_sum = by_segment ? nullptr : a.p_gate ? a.p_gate + base : nullptr;
    auto flush = [&] {                              // the segment is wholly this workgroup's: its gradient is done
        if (!by_segment || !a.p_gate || seg < 0 || a.cu[seg] < r0 || a.cu[seg + 1] > r1) return;
        for (int c = threadIdx.x; c < a.H; c += 256) {
            const size_t at = (size_t)seg * a.H + c;
            if (a.grad_f32) ((float *)a.d_gate)[at] = gate_sum[c] + (a.accumulate ? ((float *)a.d_gate)[at] : 0.f);
            else Elem<T>::store((T *)a.d_gate + at, gate_sum[c] + (a.accumulate ? Elem<T>::load((T *)a.d_gate + at) : 0.f));
        }
    };
    for (int t = r0; t < r1; ++t) {
        const size_t off = (size_t)t * a.H;
        if (by_segment && t >= seg_end) {
            flush();
            seg = find_segment(a.cu, a.S, t);
            seg_end = a.cu[seg + 1];
            if (first_seg < 0) first_seg = seg;
            gate = (const T *)a.gate_v + (size_t)seg * a.H;
            if (a.p_gate) {
                gate_sum = a.p_gate + (size_t)(2 * blockIdx.x + (seg != first_seg)) * a.H;
                for (int c = threadIdx.x; c < a.H; c += 256) gate_sum[c] = 0.f;
            }
        }
        const T *y = (const T *)a.y + off, *dh = (const T *)a.dh + off, *b = (const T *)a.b + off;
        const float mu = a.pre == NORM_LAYER ? a.pre_mean[t] : 0.f, r = a.pre != NORM_NONE ? a.pre_rstd[t] : 0.f;
        float s0 = 0.f, s1 = 0.f;
        if (a.pre != NORM_NONE) {
            for (int c = threadIdx.x; c < a.H; c += 256) {
                const float d = Elem<T>::load(dh + c), hat = (Elem<T>::load(y + c) - mu) * r, back = d * Elem<T>::load((const T *)a.pre_w + c);
                s0 += back; s1 += back * hat;
                if (a.p_pre_w) a.p_pre_w[base + c] += d * hat;
                if (a.p_pre_b) a.p_pre_b[base + c] += d;
            }
            s1 = block_sum<4>(s1, red) / a.H;
            s0 = a.pre == NORM_LAYER ? block_sum<4>(s0, red) / a.H : 0.f;
        }
        const float mu2 = a.post == NORM_LAYER ? a.post_mean[t] : 0.f, r2 = a.post != NORM_NONE ? a.post_rstd[t] : 0.f;
        float u0 = 0.f, u1 = 0.f;
        for (int c = threadIdx.x; c < a.H; c += 256) {
            float d = a.dy ? Elem<T>::load((const T *)a.dy + off + c) : 0.f;
            if (a.pre != NORM_NONE)
                d += r * (Elem<T>::load(dh + c) * Elem<T>::load((const T *)a.pre_w + c) - s0 - (Elem<T>::load(y + c) - mu) * r * s1);
            total[c] = d;
            if (!a.b) continue;
            float n = Elem<T>::load(b + c), hat = 0.f;
            if (a.post != NORM_NONE) n = hat = (n - mu2) * r2;
            const float dn = a.beta * d * (a.gate != GATE_NONE ? Elem<T>::load(gate + c) : 1.f);
            if (a.post != NORM_NONE) {
                const float w = Elem<T>::load((const T *)a.post_w + c), back = dn * w;
                n *= w;
                if (a.post == NORM_LAYER) n += Elem<T>::load((const T *)a.post_b + c);
                u0 += back; u1 += back * hat;
                if (a.p_post_w) a.p_post_w[base + c] += dn * hat;
                if (a.p_post_b) a.p_post_b[base + c] += dn;
            }
            if (gate_sum) gate_sum[c] += a.beta * n * d;
        }
        if (a.b && a.post != NORM_NONE) {
            u1 = block_sum<4>(u1, red) / a.H;
            u0 = a.post == NORM_LAYER ? block_sum<4>(u0, red) / a.H : 0.f;
        }
        for (int c = threadIdx.x; c < a.H; c += 256) {
            const float d = total[c];
            if (a.db) {
                float v = a.beta * d * (a.gate != GATE_NONE ? Elem<T>::load(gate + c) : 1.f);
                if (a.post != NORM_NONE) v = r2 * (v * Elem<T>::load((const T *)a.post_w + c) - u0 - (Elem<T>::load(b + c) - mu2) * r2 * u1);
                Elem<T>::store((T *)a.db + off + c, v);
            }
            if (a.dx) Elem<T>::store((T *)a.dx + off + c, a.b ? a.alpha * d : d);
        }
    }
    flush();
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

}  // namespace

hipError_t join_fwd(int dtype, const JoinArgs &a, hipStream_t st) {
    if (a.T == 0) return hipSuccess;
    if (dtype == DT_F32) join_fwd_kernel<float><<<a.T, 256, 0, st>>>(a);
    else join_fwd_kernel<bf16_t><<<a.T, 256, 0, st>>>(a);
    return hipGetLastError();
}

int join_bwd_blocks(int T, int) { return T < 512 ? T : 512; }

hipError_t join_bwd(int dtype, const JoinArgs &a, hipStream_t st) {
    const int blocks = join_bwd_blocks(a.T, a.H);
    if (a.T == 0 && !(a.d_gate && a.S > 0)) return hipSuccess;
    if (a.T > 0) {
        if (dtype == DT_F32) join_bwd_kernel<float><<<blocks, 256, 0, st>>>(a);
        else join_bwd_kernel<bf16_t><<<blocks, 256, 0, st>>>(a);
    }
    if (a.gate == GATE_SEGMENT && a.d_gate && a.S > 0) {
        for (int s = 0; s < a.S; s += 65535) {          // a grid's second dimension ends there
            const dim3 grid(ceil_div(a.H, 256), a.S - s < 65535 ? a.S - s : 65535);
            const size_t at = (size_t)s * a.H;
            if (a.grad_f32 || dtype == DT_F32) gate_segments_kernel<float><<<grid, 256, 0, st>>>(a.p_gate, a.cu + s, a.T, a.H, blocks, (float *)a.d_gate + at, a.accumulate);
            else gate_segments_kernel<bf16_t><<<grid, 256, 0, st>>>(a.p_gate, a.cu + s, a.T, a.H, blocks, (bf16_t *)a.d_gate + at, a.accumulate);
        }
    }
    return hipGetLastError();
}

}  // namespace mmt
