// Rotary positions of whole heads or their front part.
#include "ops.h"

namespace mmt {
namespace {

template <typename T>
__global__ __launch_bounds__(256) void rope_heads_kernel(RopeArgs a) {
    const int units = a.half + (a.x == a.y ? 0 : a.d - 2 * a.half);         // pairs, then features that pass through
    const long idx = (long)blockIdx.x * 256 + threadIdx.x;
    if (idx >= (long)a.T * a.heads * units) return;
    const int u = (int)(idx % units), h = (int)(idx / units % a.heads);
    const long t = idx / ((long)units * a.heads);
    const T *x = (const T *)a.x + t * a.ldx + (long)h * a.d;
    T *y = (T *)a.y + t * a.ldy + (long)h * a.d;
    if (u >= a.half) {
        y[u + a.half] = x[u + a.half];
        return;
    }
    const int pos = a.positions ? a.positions[t] : (int)t - a.cu[find_segment(a.cu, a.S, (int)t)];
    const double turn = pos * a.turns[u];
    float s, c;
    sincospif(2.f * (float)(turn - rint(turn)), &s, &c);
    c *= a.cos_scale; s *= a.sin_scale;
    const int i0 = a.interleaved ? 2 * u : u, i1 = a.interleaved ? 2 * u + 1 : u + a.half;
    const float v0 = Elem<T>::load(x + i0), v1 = Elem<T>::load(x + i1);
    Elem<T>::store(y + i0, v0 * c - v1 * s);
    Elem<T>::store(y + i1, v1 * c + v0 * s);
}

}  // namespace

hipError_t rope(int dtype, const RopeArgs &a, hipStream_t st) {
    const long total = (long)a.T * a.heads * (a.half + (a.x == a.y ? 0 : a.d - 2 * a.half));
    if (total == 0) return hipSuccess;
    const long blocks = (total + 255) / 256;
    if (blocks > 0x7fffffff) return hipErrorInvalidValue;
    if (dtype == DT_F32) rope_heads_kernel<float><<<(unsigned)blocks, 256, 0, st>>>(a);
    else rope_heads_kernel<bf16_t><<<(unsigned)blocks, 256, 0, st>>>(a);
    return hipGetLastError();
}

}  // namespace mmt
