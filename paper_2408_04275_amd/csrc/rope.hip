// Rotary positions of whole heads or their front part.
//
// Memory-bound: each feature is read and written once, and the 2 half numbers of a token's rotation serve all its heads.  So a
// workgroup takes whole tokens: its threads first put the rotations of its tokens into LDS (an angle in fp64 each, reduced to a
// turn, then sine and cosine in fp32), the data of their first heads already on its way, and then walk over the heads in chunks of up to 16
// bytes.  No table in memory, no launch before this one.
// bf16, out of HBM: 8192 tokens of 64 heads of 128 in place 55 us (4.8 TB/s), 16411 of 72 heads, 64 of 128 features interleaved, out of place 115 us
// (5.3 TB/s).  Streaming accesses would save a tenth of the first (50 us) and cost others up to a half (80-wide fp32 heads 16 -> 27 us): they pay only where a
// wavefront covers whole lines, and the products that read the result next find less of it in the caches.
#include "ops.h"
#include "chunk.h"
#include <algorithm>

namespace mmt {
namespace {

struct RopeShape {
    int tile;                   // tokens a workgroup
    int units;                  // chunk pairs of a head: first the rotated ones, then those that pass through
    int rot_units, copy_chunks;
    int group;                  // heads a workgroup has at work at once: 256 / units
    int step_tokens, step_heads;// group = step_tokens * heads + step_heads
};

// A unit is two chunks of V elements, and neighbouring threads' first (and second) chunks are neighbours in memory: features u V.. and half + u V.. of
// the rotated part -- V whole pairs in either layout, but for single features of interleaved pairs -- or, of the features that pass through,
// chunks k and k + their units (the last unit may have the first alone).
template <typename T, int V, bool INTERLEAVED>
__global__ __launch_bounds__(256) void rope_heads_kernel(RopeArgs a, RopeShape s) {
    extern __shared__ float2 turned[];                       // [tile][half]: cosine, sine
    const long first = (blockIdx.y * (long)gridDim.x + blockIdx.x) * s.tile;
    if (first >= a.T) return;
    const int t0 = (int)first, tokens = min(s.tile, a.T - t0);
    const int u = threadIdx.x % s.units, g = threadIdx.x / s.units;
    const bool rotates = u < s.rot_units;
    constexpr bool SINGLE = INTERLEAVED && V == 1;
    const int copy = u - s.rot_units, copy_units = s.units - s.rot_units;
    const int o0 = rotates ? (SINGLE ? 2 * u : u * V) : 2 * a.half + copy * V;
    const int o1 = rotates ? (SINGLE ? o0 + 1 : o0 + a.half) : o0 + copy_units * V;
    const bool second = rotates || copy + copy_units < s.copy_chunks;
    int tok = g / a.heads, head = g % a.heads;
    const bool active = g < s.group;
    Chunk<T, V> c0, c1;
    auto request = [&] {
        const T *x = (const T *)a.x + (t0 + tok) * a.ldx + (long)head * a.d;
        c0.load(x + o0);
        if (second) c1.load(x + o1);
    };
    if (active && tok < tokens) request();
    for (int k = threadIdx.x; k < tokens * a.half; k += 256) {
        const int t = t0 + k / a.half;
        const int pos = a.positions ? a.positions[t] : t - a.cu[find_segment(a.cu, a.S, t)];
        const double turn = pos * a.turns[k % a.half];
        float si, co;
        sincospif(2.f * (float)(turn - rint(turn)), &si, &co);
        turned[k] = make_float2(co * a.cos_scale, si * a.sin_scale);
    }
    __syncthreads();
    if (!active) return;
    while (tok < tokens) {
        T *y = (T *)a.y + (t0 + tok) * a.ldy + (long)head * a.d;
        const float2 *cs = turned + tok * a.half;
        Chunk<T, V> d0 = c0, d1 = c1;
        tok += s.step_tokens; head += s.step_heads;
        if (head >= a.heads) { head -= a.heads; ++tok; }
        if (tok < tokens) request();
        if (rotates) {
            float lo[V], hi[V];
#pragma unroll
            for (int i = 0; i < V; ++i) { lo[i] = d0.get(i); hi[i] = d1.get(i); }
            auto turn = [](float &p, float &q, float2 r) {
                const float v = p;
                p = v * r.x - q * r.y;
                q = q * r.x + v * r.y;
            };
            if constexpr (INTERLEAVED && !SINGLE) {
#pragma unroll
                for (int i = 0; i < V; i += 2) {
                    turn(lo[i], lo[i + 1], cs[(o0 + i) / 2]);
                    turn(hi[i], hi[i + 1], cs[(o1 + i) / 2]);
                }
            } else {
#pragma unroll
                for (int i = 0; i < V; ++i) turn(lo[i], hi[i], cs[u * V + i]);
            }
            d0.set(lo); d1.set(hi);
        }
        d0.store(y + o0);
        if (second) d1.store(y + o1);
    }
}

template <typename T, int V>
hipError_t launch(const RopeArgs &a, hipStream_t st) {
    RopeShape s;
    s.rot_units = a.half / V;
    s.copy_chunks = a.x == a.y ? 0 : (a.d - 2 * a.half) / V;
    s.units = s.rot_units + (s.copy_chunks + 1) / 2;         // at most 128
    s.group = 256 / s.units;
    s.step_tokens = s.group / a.heads;
    s.step_heads = s.group % a.heads;
    // Tokens a workgroup: two units a thread, and not so many that a short call leaves the chip idle or that LDS fills up.  More tokens share nothing but
    // the start: 16411 tokens of 72 heads, 8 -> 1 a workgroup 133 -> 115 us; fewer leave threads without work (12000 tokens of 12 heads, 20 features each,
    // 5 -> 1 10.5 -> 15.6 us).
    const int by_units = (511 + a.heads * s.units) / (a.heads * s.units), by_angles = 1024 / a.half, by_tokens = a.T / 512;
    s.tile = std::max(1, std::min({by_units, by_angles, by_tokens}));
    const size_t lds = (size_t)s.tile * a.half * sizeof(float2);
    // a grid's first dimension ends at 2^32 threads
    const int blocks = ceil_div(a.T, s.tile);
    const dim3 grid(std::min(blocks, 1 << 20), ceil_div(blocks, 1 << 20));
    if (a.interleaved) rope_heads_kernel<T, V, true><<<grid, 256, lds, st>>>(a, s);
    else rope_heads_kernel<T, V, false><<<grid, 256, lds, st>>>(a, s);
    return hipGetLastError();
}

}  // namespace

hipError_t rope(int dtype, const RopeArgs &a, hipStream_t st) {
    if (a.T == 0) return hipSuccess;
    // elements that every chunk's place is a multiple of: the widest chunk that all accesses are aligned for.  12000 bf16 tokens of 40 heads of 80, us, of which
    // 20 / 40 / 80 features rotate (chunks of 4 / 8 / 16 bytes): in place 33.7 / 37.2 / 36.6: the heads' whole lines are read
    // whatever rotates, so narrow chunks cost nothing; out of place 50.5 / 38.4 / 36.1, where the features that pass through go by the narrow chunks too
    const long places = a.half | a.d | a.ldx | a.ldy;
    const int v = dtype == DT_F32 ? (places % 4 == 0 ? 4 : places % 2 == 0 ? 2 : 1)
                                  : (places % 8 == 0 ? 8 : places % 4 == 0 ? 4 : places % 2 == 0 ? 2 : 1);
    if (dtype == DT_F32) return v == 4 ? launch<float, 4>(a, st) : v == 2 ? launch<float, 2>(a, st) : launch<float, 1>(a, st);
    return v == 8 ? launch<bf16_t, 8>(a, st) : v == 4 ? launch<bf16_t, 4>(a, st) : v == 2 ? launch<bf16_t, 2>(a, st) : launch<bf16_t, 1>(a, st);
}

}  // namespace mmt
