// Attention of runs of queries to ranges of keys in fp32 on the fp32 matrix instruction (v_mfma_f32_16x16x4_f32), forward and backward: the
// rows, tiles and zeros of cross_mfma.hip with blocks of 16.
//
// A workgroup owns 16 rows of a run (forward, dQ) or 16 keys (dK/dV) of one key/value head; its wavefronts share out the 16-row blocks of
// the other side, and their partial results are combined through LDS in a fixed order.  As in attn_f32.hip a lane holds one owned row
// (lane & 15) and the four streamed rows 4 (lane >> 4) .. + 3 of a score tile, and operands come straight from global memory in two
// forms: a row's 16-byte pieces where the features are contracted (feature 16 b + 4 (lane >> 4) + j for MFMA j of block b), and features of a row
// across the lanes where they are the result's rows: of whole 64s four neighbouring ones per lane (fragment 4 c + f holds features 64 c + 4 x + f), of what is left
// one (fragment 4 C + r holds features 64 C + 16 r + x).  Heads are KB blocks of 16 features wide.
#include "cross_tiles.h"
#include <algorithm>

namespace mmt {

namespace {

__device__ __forceinline__ f32x4 mfma(float a, float b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x4f32(a, b, c, 0, 0, 0); }
__device__ __forceinline__ f32x4 load4(__amdgpu_buffer_rsrc_t rs, uint32_t off) {
    const u32x4 w = __builtin_amdgcn_raw_buffer_load_b128(rs, (int)off, 0, 0);
    return *reinterpret_cast<const f32x4 *>(&w);
}
constexpr uint32_t NO_ROW = 0x80000000u;                // behind every buffer's end

template <int KB> struct Pieces { f32x4 v[KB]; };       // features contracted
template <int KB> struct Columns {                      // rows contracted
    static constexpr int C = KB / 4, R = KB % 4;
    f32x4 wide[4][C > 0 ? C : 1];
    float one[4][R > 0 ? R : 1];
};

// 16 rows of a tensor, by the byte offset of each (NO_ROW: it reads as zeros)
struct Block {
    __amdgpu_buffer_rsrc_t rs;
    uint32_t row;               // of row lane & 15
    uint32_t quad[4];           // of rows 4 (lane >> 4) ..
};
template <int KB>
__device__ __forceinline__ void pieces(const Block &b, Pieces<KB> &p) {
    const uint32_t o = b.row + ((threadIdx.x & 48) >> 4) * 16u;
#pragma unroll
    for (int i = 0; i < KB; ++i) p.v[i] = load4(b.rs, o + 64u * i);
}
template <int KB>
__device__ __forceinline__ void columns(const Block &b, Columns<KB> &c) {
    const uint32_t x = threadIdx.x & 15;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
#pragma unroll
        for (int i = 0; i < Columns<KB>::C; ++i) c.wide[j][i] = load4(b.rs, b.quad[j] + 16u * x + 256u * i);
#pragma unroll
        for (int i = 0; i < Columns<KB>::R; ++i)
            c.one[j][i] = __uint_as_float(__builtin_amdgcn_raw_buffer_load_b32(b.rs, (int)(b.quad[j] + 4u * x + 256u * Columns<KB>::C + 64u * i), 0, 0));
    }
}
// keys key .. of a tensor of keys, those below end
__device__ __forceinline__ Block key_block(const float *p, long ld, int dh, int key, int end) {
    Block b;
    const int n = min(end - key, 16);
    const uint32_t bytes = n > 0 ? (uint32_t)((n - 1) * (int)ld + dh) * 4u : 0u;
    b.rs = __builtin_amdgcn_make_buffer_rsrc(const_cast<float *>(p + key * ld), 0, (int)bytes, 0x00020000);
    const int x = threadIdx.x & 15, q4 = ((threadIdx.x & 48) >> 4) * 4;
    b.row = x < n ? (uint32_t)(x * (int)ld) * 4u : NO_ROW;
#pragma unroll
    for (int j = 0; j < 4; ++j) b.quad[j] = q4 + j < n ? (uint32_t)((q4 + j) * (int)ld) * 4u : NO_ROW;
    return b;
}
// rows of a run
__device__ __forceinline__ Block row_block(const float *p, long ld, int dh, const Rows &at, const Group &g) {
    Block b;
    b.rs = __builtin_amdgcn_make_buffer_rsrc(const_cast<float *>(p + at.t * ld), 0, 0x7fff0000, 0x00020000);
    const int x = threadIdx.x & 15, q4 = ((threadIdx.x & 48) >> 4) * 4;
    const uint32_t row = at.offset(g, x, ld, dh) * 4u;
    b.row = x < at.left ? row : NO_ROW;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const uint32_t quad = at.offset(g, q4 + j, ld, dh) * 4u;
        b.quad[j] = q4 + j < at.left ? quad : NO_ROW;
    }
    return b;
}

// score-shaped product: [streamed row 4 (lane >> 4) + e][owned row lane & 15]
template <int KB>
__device__ __forceinline__ f32x4 dot_rows(const Pieces<KB> &streamed, const Pieces<KB> &owned) {
    f32x4 s[2] = {f32x4{0.f, 0.f, 0.f, 0.f}, f32x4{0.f, 0.f, 0.f, 0.f}};       // two chains: an MFMA's result is several cycles away
#pragma unroll
    for (int b = 0; b < KB; ++b)
#pragma unroll
        for (int j = 0; j < 4; ++j) s[j & 1] = mfma(streamed.v[b][j], owned.v[b][j], s[j & 1]);
    return s[0] + s[1];
}
// acc[feature][owned row] += sum over the 16 streamed rows of x[row][feature] * w[row][owned row]
template <int KB>
__device__ __forceinline__ void add_rows(f32x4 (&acc)[KB], const Columns<KB> &x, const f32x4 &w) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
#pragma unroll
        for (int c = 0; c < Columns<KB>::C; ++c)
#pragma unroll
            for (int f = 0; f < 4; ++f) acc[4 * c + f] = mfma(x.wide[j][c][f], w[j], acc[4 * c + f]);
#pragma unroll
        for (int r = 0; r < Columns<KB>::R; ++r) acc[4 * Columns<KB>::C + r] = mfma(x.one[j][r], w[j], acc[4 * Columns<KB>::C + r]);
    }
}

// a lane's share of the [owned row][feature] result, handed to out(row, first of four features, value)
template <int KB, typename F>
__device__ __forceinline__ void lane_parts(const f32x4 (&acc)[KB], F out) {
    const int r = threadIdx.x & 15, q = (threadIdx.x & 48) >> 4;
    constexpr int C = Columns<KB>::C;
#pragma unroll
    for (int c = 0; c < C; ++c)
#pragma unroll
        for (int e = 0; e < 4; ++e) out(r, 64 * c + 16 * q + 4 * e, f32x4{acc[4 * c][e], acc[4 * c + 1][e], acc[4 * c + 2][e], acc[4 * c + 3][e]});
#pragma unroll
    for (int i = 0; i < Columns<KB>::R; ++i) out(r, 64 * C + 16 * i + 4 * q, acc[4 * C + i]);
}

// the wavefronts' [16 owned rows][D] results
template <int KB, int NW>
struct Partials {
    static constexpr int D = 16 * KB, PITCH = D + 4;
    float v[NW][16][PITCH];
    __device__ __forceinline__ void put(int wave, const f32x4 (&acc)[KB]) {
        lane_parts(acc, [&](int row, int col, f32x4 x) { *reinterpret_cast<f32x4 *>(&v[wave][row][col]) = x; });
    }
    // sums times `scale`, handed to out(row, first of four features, value)
    template <typename F>
    __device__ __forceinline__ void each(float scale, F out) const {
        for (int i = threadIdx.x; i < 16 * D / 4; i += 64 * NW) {
            const int row = i / (D / 4), col = i % (D / 4) * 4;
            f32x4 s = *reinterpret_cast<const f32x4 *>(&v[0][row][col]);
#pragma unroll
            for (int w = 1; w < NW; ++w) s += *reinterpret_cast<const f32x4 *>(&v[w][row][col]);
            out(row, col, s * scale);
        }
    }
};

__device__ __forceinline__ float row_sum(float v) { v += __shfl_xor(v, 16, 64); return v + __shfl_xor(v, 32, 64); }
__device__ __forceinline__ float row_max(float v) { v = fmaxf(v, __shfl_xor(v, 16, 64)); return fmaxf(v, __shfl_xor(v, 32, 64)); }

template <int KB, int NW>
__global__ __launch_bounds__(64 * NW) void cross_f32_fwd_kernel(CrossArgs a) {
    __shared__ __attribute__((aligned(16))) Partials<KB, NW> part;
    __shared__ float stat_m[NW][16], stat_l[NW][16];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r = threadIdx.x & 15, q4 = ((threadIdx.x & 48) >> 4) * 4;
    const int head = blockIdx.x % a.nkv, dh = a.d;
    const Item it = find_item(a, blockIdx.x / a.nkv, 16, a.chunk);
    const int parts = a.chunk ? max((it.hi - it.lo + a.chunk - 1) / a.chunk, 1) : 1;
    const Group g(a);
    const Rows mine(it, g, it.index / parts * 16);
    const int kbeg = it.lo + it.index % parts * a.chunk, kend = parts > 1 ? min(kbeg + a.chunk, it.hi) : it.hi;
    const float *const K = (const float *)a.k + (long)head * dh, *const V = (const float *)a.v + (long)head * dh;
    Pieces<KB> q;
    pieces(row_block((const float *)a.q + (long)head * g.n * dh, a.ldq, dh, mine, g), q);
    f32x4 acc[KB];
#pragma unroll
    for (int i = 0; i < KB; ++i) acc[i] = f32x4{0.f, 0.f, 0.f, 0.f};
    float m = -INFINITY, l = 0.f;
    for (int k0 = kbeg + 16 * wave; k0 < kend; k0 += 16 * NW) {
        Pieces<KB> k;
        Columns<KB> v;
        pieces(key_block(K, a.ldk, dh, k0, kend), k);
        columns(key_block(V, a.ldv, dh, k0, kend), v);
        f32x4 p = dot_rows(k, q) * a.scale;
        float mx = -INFINITY;
#pragma unroll
        for (int e = 0; e < 4; ++e) { if (k0 + q4 + e >= kend) p[e] = -INFINITY; mx = fmaxf(mx, p[e]); }
        const float mn = fmaxf(m, row_max(mx)), base = mn == -INFINITY ? 0.f : mn, corr = expf(m - base);
        l *= corr;
#pragma unroll
        for (int e = 0; e < 4; ++e) { p[e] = expf(p[e] - base); l += p[e]; }
#pragma unroll
        for (int i = 0; i < KB; ++i) acc[i] *= corr;
        m = mn;
        add_rows(acc, v, p);
    }
    l = row_sum(l);
    if (threadIdx.x % 64 < 16) { stat_m[wave][r] = m; stat_l[wave][r] = l; }
    __syncthreads();
    float top = stat_m[0][r], total = 0.f;
#pragma unroll
    for (int w = 1; w < NW; ++w) top = fmaxf(top, stat_m[w][r]);
    const float base = top == -INFINITY ? 0.f : top;
#pragma unroll
    for (int w = 0; w < NW; ++w) total += stat_l[w][r] * expf(stat_m[w][r] - base);
    const float f = expf(m - base) * (parts > 1 ? 1.f : total > 0.f ? 1.f / total : 0.f);
#pragma unroll
    for (int i = 0; i < KB; ++i) acc[i] *= f;
    part.put(wave, acc);
    __syncthreads();
    if (parts > 1) {
        float *out = a.part + (size_t)blockIdx.x * 16 * dh;
        part.each(1.f, [&](int row, int col, f32x4 v) { if (row < mine.left) *reinterpret_cast<f32x4 *>(out + row * dh + col) = v; });
        if (threadIdx.x < 16 && r < mine.left) a.part_ml[(size_t)blockIdx.x * 16 + r] = make_float2(top, total);
        return;
    }
    float *out = (float *)a.o + mine.t * a.ldo + (long)head * g.n * dh;
    part.each(1.f, [&](int row, int col, f32x4 v) { if (row < mine.left) *reinterpret_cast<f32x4 *>(out + mine.offset(g, row, a.ldo, dh) + col) = v; });
    if (a.lse && threadIdx.x < 16 && r < mine.left) {
        const int tok = g.token(mine.j + r), h = head * g.n + mine.j + r - tok * g.n;
        a.lse[(long)h * a.Tq + mine.t + tok] = top + logf(total);
    }
}

// The chunks' results of 16 rows, by the workgroup of chunk 0
__global__ __launch_bounds__(256) void cross_f32_combine_kernel(CrossArgs a) {
    const int head = blockIdx.x % a.nkv, dh = a.d;
    const Item it = find_item(a, blockIdx.x / a.nkv, 16, a.chunk);
    const int parts = max((it.hi - it.lo + a.chunk - 1) / a.chunk, 1);
    if (parts == 1 || it.index % parts) return;
    const Group g(a);
    const Rows mine(it, g, it.index / parts * 16);
    const int quads = dh / 4, rows = min(mine.left, 16);
    const size_t stride = (size_t)a.nkv * 16;
    for (int e = threadIdx.x; e < rows * quads; e += 256) {
        const int r = e / quads, c = e % quads * 4;
        const float2 *ml = a.part_ml + (size_t)blockIdx.x * 16 + r;
        const float *part = a.part + ((size_t)blockIdx.x * 16 + r) * dh + c;
        float m = -INFINITY, l = 0.f;
        f32x4 x = {0.f, 0.f, 0.f, 0.f};
        for (int j0 = 0; j0 < parts; j0 += 8) {
            float2 v[8];
            f32x4 y[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                v[i] = make_float2(-INFINITY, 0.f);
                y[i] = f32x4{0.f, 0.f, 0.f, 0.f};
                if (j0 + i < parts) {
                    v[i] = ml[(j0 + i) * stride];
                    y[i] = *reinterpret_cast<const f32x4 *>(part + (j0 + i) * stride * dh);
                }
            }
            float top = m;
#pragma unroll
            for (int i = 0; i < 8; ++i) top = fmaxf(top, v[i].x);
            const float base = top == -INFINITY ? 0.f : top, corr = expf(m - base);
            l *= corr;
            x *= corr;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float w = expf(v[i].x - base);
                l += v[i].y * w;
                x += y[i] * w;
            }
            m = top;
        }
        const int tok = g.token(mine.j + r), h = head * g.n + mine.j + r - tok * g.n;
        *reinterpret_cast<f32x4 *>((float *)a.o + (mine.t + tok) * a.ldo + (long)h * dh + c) = x * (l > 0.f ? 1.f / l : 0.f);
        if (a.lse && c == 0) a.lse[(long)h * a.Tq + mine.t + tok] = m + logf(l);
    }
}

// 1031 tokens of 16 heads of 80 in five runs of 420 keys: dQ 47 us, dK and dV 63, two fifths of the matrix rate; larger packs reach 60 % of it.  Each operand is loaded by the
// wavefront that uses it, twice where it is a row of both products, in several rounds of loads and waits an iteration; more registers for loads ahead leave fewer
// wavefronts (dQ 50 us).
// Four wavefronts a SIMD (left to the compiler 1 to 10 % slower: 294 rows of 16 heads of 64 in runs that see 29760 keys 110 -> 99 us).
// dQ_i = scale * sum_j dS_ij k_j,  dS_ij = P_ij (dO_i . v_j - D_i),  D_i = dO_i . O_i (kept in a.D),  P_ij = exp(s_ij - lse_i)
template <int KB, int NW>
__global__ __launch_bounds__(64 * NW) __attribute__((amdgpu_waves_per_eu(KB <= 5 ? 4 : 1, KB <= 5 ? 4 : 8))) void cross_f32_dq_kernel(CrossArgs a) {
    __shared__ __attribute__((aligned(16))) union { Partials<KB, NW> part; int plan[PLAN_LDS / 4]; } lds;
    Partials<KB, NW> &part = lds.part;
    int block = blockIdx.x;
    if (a.n_tiles > 0 && block-- == 0) { make_plan<64 * NW>(a, lds.plan); return; }
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r = threadIdx.x & 15, q4 = ((threadIdx.x & 48) >> 4) * 4;
    const int head = block % a.nkv, dh = a.d;
    const Item it = find_item(a, block / a.nkv, 16, a.chunk);
    const int parts = a.chunk ? max((it.hi - it.lo + a.chunk - 1) / a.chunk, 1) : 1;
    const Group g(a);
    const Rows mine(it, g, it.index / parts * 16);
    const int kbeg = it.lo + it.index % parts * a.chunk, kend = parts > 1 ? min(kbeg + a.chunk, it.hi) : it.hi;
    const long col = (long)head * g.n * dh;
    const float *const K = (const float *)a.k + (long)head * dh, *const V = (const float *)a.v + (long)head * dh;
    Pieces<KB> q, go, o;
    pieces(row_block((const float *)a.q + col, a.ldq, dh, mine, g), q);
    pieces(row_block((const float *)a.d_o + col, a.lddo, dh, mine, g), go);
    pieces(row_block((const float *)a.o + col, a.ldo, dh, mine, g), o);
    float D = 0.f, lse = 0.f;
#pragma unroll
    for (int i = 0; i < KB; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) D += go.v[i][e] * o.v[i][e];
    D = row_sum(D);
    if (r < mine.left) {
        const int tok = g.token(mine.j + r), h = head * g.n + mine.j + r - tok * g.n;
        const long at = (long)h * a.Tq + mine.t + tok;
        lse = a.lse[at];
        if (threadIdx.x < 16 && kbeg == it.lo) a.D[at] = D;
    }
    if (!a.dq) return;
    f32x4 acc[KB];
#pragma unroll
    for (int i = 0; i < KB; ++i) acc[i] = f32x4{0.f, 0.f, 0.f, 0.f};
    for (int k0 = kbeg + 16 * wave; k0 < kend; k0 += 16 * NW) {
        Pieces<KB> k, v;
        Columns<KB> kc;
        const Block kb = key_block(K, a.ldk, dh, k0, kend);
        pieces(kb, k);
        pieces(key_block(V, a.ldv, dh, k0, kend), v);
        columns(kb, kc);
        const f32x4 s = dot_rows(k, q) * a.scale, dp = dot_rows(v, go);
        f32x4 ds;
#pragma unroll
        for (int e = 0; e < 4; ++e) ds[e] = k0 + q4 + e < kend ? expf(s[e] - lse) * (dp[e] - D) : 0.f;
        add_rows(acc, kc, ds);
    }
    part.put(wave, acc);
    __syncthreads();
    if (parts > 1) {
        float *out = a.part + (size_t)block * 16 * dh;
        part.each(1.f, [&](int row, int c, f32x4 v) { if (row < mine.left) *reinterpret_cast<f32x4 *>(out + row * dh + c) = v; });
        return;
    }
    float *out = (float *)a.dq + mine.t * a.lddq + col;
    part.each(a.scale, [&](int row, int c, f32x4 v) { if (row < mine.left) *reinterpret_cast<f32x4 *>(out + mine.offset(g, row, a.lddq, dh) + c) = v; });
}

// dK_j = scale * sum_i dS_ij q_i,   dV_j = sum_i P_ij dO_i over the rows i of the runs that see the keys
// OWN: each wavefront has 16 keys to itself and walks all rows, without LDS; up to 64 features three wavefronts a SIMD (us, left to the compiler / three: 1000 rows
// of 16 heads in eight runs of 1000 keys 124 / 120, 294 in runs that see 29760 keys 167 / 163; with 80 features 51.5 / 55).
template <int KB, int NW, bool OWN>
__global__ __launch_bounds__(64 * NW) __attribute__((amdgpu_waves_per_eu(OWN && KB <= 4 ? 3 : 1, OWN && KB <= 4 ? 3 : 8))) void cross_f32_dkv_kernel(CrossArgs a) {
    __shared__ __attribute__((aligned(16))) std::conditional_t<OWN, int, Partials<KB, NW>> part;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), q4 = ((threadIdx.x & 48) >> 4) * 4;
    const int head = blockIdx.x % a.nkv, dh = a.d, block = blockIdx.x / a.nkv;
    constexpr int BLOCKS = TILE_KEYS / 16 / (OWN ? NW : 1);          // workgroups of a tile
    KeyTile kt = find_tile(a, block / BLOCKS);
    kt.key += (OWN ? block % BLOCKS * NW + wave : block % BLOCKS) * 16;
    if (kt.key >= kt.end) return;
    const Group g(a);
    const long col = (long)head * g.n * dh;
    Pieces<KB> k, v;
    pieces(key_block((const float *)a.k + (long)head * dh, a.ldk, dh, kt.key, kt.end), k);
    pieces(key_block((const float *)a.v + (long)head * dh, a.ldv, dh, kt.key, kt.end), v);
    f32x4 dk[KB], dv[KB];
#pragma unroll
    for (int i = 0; i < KB; ++i) dk[i] = dv[i] = f32x4{0.f, 0.f, 0.f, 0.f};
    // blocks of 16 rows: the first of all steps, then the second ... (of short runs no more than the first exists)
    for (int i = OWN ? 0 : wave; i < 4 * kt.steps; i += OWN ? 1 : NW) {
        const int quarter = (i >= kt.steps) + (i >= 2 * kt.steps) + (i >= 3 * kt.steps);
        const Rows step = rows_of(entry_of(a.steps, kt.step + i - quarter * kt.steps));
        Rows at;
        const int first = step.j + quarter * 16, tok = g.token(first);
        at.t = step.t + tok; at.j = first - tok * g.n; at.left = step.left - quarter * 16;
        if (at.left <= 0) continue;
        f32x4 lse, D;
        const long first_head = (long)head * g.n * a.Tq + at.t;
        const __amdgpu_buffer_rsrc_t lses = __builtin_amdgcn_make_buffer_rsrc(a.lse + first_head, 0, 0x7fff0000, 0x00020000),
                                     Ds = __builtin_amdgcn_make_buffer_rsrc(a.D + first_head, 0, 0x7fff0000, 0x00020000);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int t = g.token(at.j + q4 + e), h = at.j + q4 + e - t * g.n;
            const uint32_t there = (uint32_t)(h * a.Tq + t) * 4u, off = q4 + e < at.left ? there : NO_ROW;
            lse[e] = __uint_as_float(__builtin_amdgcn_raw_buffer_load_b32(lses, (int)off, 0, 0));
            D[e] = __uint_as_float(__builtin_amdgcn_raw_buffer_load_b32(Ds, (int)off, 0, 0));
        }
        Pieces<KB> q, go;
        Columns<KB> qc, gc;
        const Block qb = row_block((const float *)a.q + col, a.ldq, dh, at, g), gb = row_block((const float *)a.d_o + col, a.lddo, dh, at, g);
        pieces(qb, q);
        pieces(gb, go);
        columns(qb, qc);
        columns(gb, gc);
        f32x4 p, ds;
        const f32x4 s = dot_rows(q, k) * a.scale, dp = dot_rows(go, v);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            p[e] = q4 + e < at.left ? expf(s[e] - lse[e]) : 0.f;
            ds[e] = q4 + e < at.left ? p[e] * (dp[e] - D[e]) : 0.f;
        }
        add_rows(dv, gc, p);
        add_rows(dk, qc, ds);
    }
    const int rows = kt.end - kt.key;
    auto store = [&](const f32x4 (&acc)[KB], void *p, long ld, float scale) {
        float *out = (float *)p + kt.key * ld + (long)head * dh;
        auto to = [&](int row, int c, f32x4 x) { if (row < rows) *reinterpret_cast<f32x4 *>(out + row * ld + c) = x; };
        if constexpr (OWN) {
            lane_parts(acc, [&](int row, int c, f32x4 x) { to(row, c, x * scale); });
        } else {
            __syncthreads();
            part.put(wave, acc);
            __syncthreads();
            part.each(scale, to);
        }
    };
    if (!OWN && a.parts > 1) {
        const int nk = a.nkv * dh;
        float *const out = a.dkv_part + (size_t)blockIdx.y * a.Tk * 2 * nk;
        store(dk, out, 2 * nk, 1.f);
        store(dv, out + nk, 2 * nk, 1.f);
        return;
    }
    store(dk, a.dk, a.lddk, a.scale);
    store(dv, a.dv, a.lddv, 1.f);
}

// eight wavefronts for heads of up to 64 features; four for wider ones, whose partial results are as large
template <int KB> constexpr int WAVES = KB <= 4 ? 8 : 4;

// f(number of blocks of 16 features)
template <typename F>
hipError_t by_width(int d, F f) {
    switch (d / 16) {
        case 1: return f(std::integral_constant<int, 1>{});
        case 2: return f(std::integral_constant<int, 2>{});
        case 3: return f(std::integral_constant<int, 3>{});
        case 4: return f(std::integral_constant<int, 4>{});
        case 5: return f(std::integral_constant<int, 5>{});
        case 6: return f(std::integral_constant<int, 6>{});
        case 7: return f(std::integral_constant<int, 7>{});
        default: return f(std::integral_constant<int, 8>{});
    }
}

}  // namespace

hipError_t cross_f32_fwd(const CrossArgs &a, const CrossPlan &p, hipStream_t st) {
    return by_width(a.d, [&](auto KB_) {
        constexpr int KB = decltype(KB_)::value;
        cross_f32_fwd_kernel<KB, WAVES<KB>><<<p.items * a.nkv, 64 * WAVES<KB>, 0, st>>>(a);
        if (a.chunk) cross_f32_combine_kernel<<<p.items * a.nkv, 256, 0, st>>>(a);
        return hipGetLastError();
    });
}

hipError_t cross_f32_bwd(const CrossArgs &a, const CrossBwdPlan &p, hipStream_t st) {
    return by_width(a.d, [&](auto KB_) {
        constexpr int KB = decltype(KB_)::value;
        if (p.items || a.n_tiles) cross_f32_dq_kernel<KB, WAVES<KB>><<<p.items * a.nkv + (a.n_tiles > 0), 64 * WAVES<KB>, 0, st>>>(a);
        if (a.chunk) cross_dq_sum_kernel<float, 16><<<p.items * a.nkv, 256, 0, st>>>(a);
        if (!a.n_tiles) return hipGetLastError();
        if (p.own) cross_f32_dkv_kernel<KB, 4, true><<<a.n_tiles * (TILE_KEYS / 64) * a.nkv, 256, 0, st>>>(a);
        else cross_f32_dkv_kernel<KB, WAVES<KB>, false><<<dim3(a.n_tiles * (TILE_KEYS / 16) * a.nkv, a.parts), 64 * WAVES<KB>, 0, st>>>(a);
        if (a.parts > 1) cross_dkv_sum_kernel<float><<<ceil_div((long)a.Tk * (2 * a.nkv * a.d / 4), 256), 256, 0, st>>>(a);
        return hipGetLastError();
    });
}

}  // namespace mmt
