// What the forward and backward kernels of cross attention have in common (see cross_mfma.hip).
#pragma once
#include "ops.h"
#include "attn_tiles.h"
#include <atomic>

namespace mmt {

namespace {

constexpr int KEYS = 64;                                // a step of the kernels with many rows
constexpr int FEW_ROWS = 32;                            // rows of a workgroup of the form for few
constexpr int STEP_ROWS = 64, TILE_KEYS = 128;          // dK/dV: rows of a step, keys of a tile
template <int D> constexpr int ROWS32 = 32 * D * 2;     // bytes of 32 rows in LDS
template <int D> constexpr int STAGE = 32 * (2 * D + 16);

// all but the N youngest LDS reads that are written as assembly have landed, x's among them
template <int N, typename V>
__device__ __forceinline__ void lds_wait(V &x) { asm volatile("s_waitcnt lgkmcnt(%1)" : "+v"(x) : "n"(N)); }

// ---- which rows and keys a workgroup has ----------------------------------------------------------------------------
__host__ __device__ inline int items_of(int tokens, int keys, int group, int tile_rows, int chunk) {
    const int tiles = (tokens * group + tile_rows - 1) / tile_rows, parts = chunk ? (keys + chunk - 1) / chunk : 1;
    return tiles * (parts > 0 ? parts : 1);
}

struct Item {
    int q0, rows, lo, hi;       // run: first token, rows of a key/value head, keys
    int index, first;           // the item's number within its run; of the run's first item among all
};

// Item y of all runs' items.  Up to 64 runs: one per lane, their items added up across the wavefront; more: from the table that
// cross_prefix_kernel left.
__device__ __forceinline__ Item find_item(const CrossArgs &a, int y, int tile_rows, int chunk) {
    const int group = a.nh / a.nkv, lane = threadIdx.x & 63;
    Item it;
    if (a.S <= 64) {
        int c0 = 0, c1 = 0, lo = 0, hi = 0;
        if (lane < a.S) { c0 = a.cu[lane]; c1 = a.cu[lane + 1]; lo = a.begin[lane]; hi = a.end[lane]; }
        const int n = lane < a.S ? items_of(c1 - c0, hi - lo, group, tile_rows, chunk) : 0;
        int sum = n;
#pragma unroll
        for (int o = 1; o < 64; o *= 2) {
            const int v = __shfl_up(sum, o, 64);
            if (lane >= o) sum += v;
        }
        const int s = min(__popcll(__builtin_amdgcn_ballot_w64(sum <= y)), 63);
        it.q0 = __builtin_amdgcn_readlane(c0, s);
        it.rows = (__builtin_amdgcn_readlane(c1, s) - it.q0) * group;
        it.lo = __builtin_amdgcn_readlane(lo, s);
        it.hi = __builtin_amdgcn_readlane(hi, s);
        it.first = __builtin_amdgcn_readlane(sum - n, s);
    } else {
        const int s = __builtin_amdgcn_readfirstlane(find_segment(a.prefix, a.S, y));
        it.q0 = __builtin_amdgcn_readfirstlane(a.cu[s]);
        it.rows = (__builtin_amdgcn_readfirstlane(a.cu[s + 1]) - it.q0) * group;
        it.lo = __builtin_amdgcn_readfirstlane(a.begin[s]);
        it.hi = __builtin_amdgcn_readfirstlane(a.end[s]);
        it.first = __builtin_amdgcn_readfirstlane(a.prefix[s]);
    }
    it.index = y - it.first;
    return it;
}

// Division of a small number (below group + 128) by the group: a product's high half (exact while number * group < 2^32)
struct Group {
    int n;
    uint32_t magic;
    __device__ __forceinline__ explicit Group(int n_) : n(n_), magic(0xffffffffu / (uint32_t)n_ + 1u) {}
    __device__ __forceinline__ explicit Group(const CrossArgs &a) : Group(a.nh / a.nkv) {}
    __device__ __forceinline__ int token(int r) const { return n == 1 ? r : (int)__umulhi((uint32_t)r, magic); }
};

// 32 rows of a run from row0 on: row i is token t + token(j + i), head of the group (j + i) % group
struct Rows {
    int t, j, left;             // first token, its first head, rows that exist
    Rows() = default;
    __device__ __forceinline__ Rows(const Item &it, const Group &g, int row0) {
        const int tok = row0 / g.n;
        t = it.q0 + tok;
        j = row0 - tok * g.n;
        left = it.rows - row0;
    }
    // elements from the first token's row of the group (stride ld, heads d wide)
    __device__ __forceinline__ uint32_t offset(const Group &g, int i, long ld, int d) const {
        const int tok = g.token(j + i);
        return (uint32_t)(tok * (int)ld + (j + i - tok * g.n) * d);
    }
};

// n rows of dh features: what stands behind them reads as zero
__device__ __forceinline__ __amdgpu_buffer_rsrc_t rows_rsrc(const bf16_t *p, long row, long ld, int n, int dh) {
    const uint32_t bytes = n > 0 ? (uint32_t)((min(n, 64) - 1) * (int)ld + dh) * 2u : 0u;
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<bf16_t *>(p + row * ld), 0, (int)bytes, 0x00020000);
}

// Copies 32 rows (`at`, of a tensor with stride ld whose group of heads starts at p) into LDS, row-major and swizzled
template <int D>
__device__ __forceinline__ void copy_rows(const bf16_t *p, long ld, int dh, const Rows &at, const Group &g, uint8_t *to) {
    constexpr int UPR = D / 8, PER = 1024 / (2 * D), N = ROWS32<D> / 1024;
    const __amdgpu_buffer_rsrc_t rs = __builtin_amdgcn_make_buffer_rsrc(const_cast<bf16_t *>(p + at.t * ld), 0, 0x7fff0000, 0x00020000);
    const int lane = threadIdx.x & 63, lrow = lane / UPR, pos = lane % UPR;
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const int row = i * PER + lrow, unit = pos ^ swz_unit<D>(row);
        const uint32_t off = row < at.left && unit * 8 < dh ? (at.offset(g, row, ld, dh) + unit * 8) * 2u : 0x80000000u;
        __builtin_amdgcn_raw_ptr_buffer_load_lds(rs, (lds_void *)(to + i * PER * 2 * D), 16, (int)off, 0, 0, 0);
    }
}

// 32 x D results of a wavefront (a lane holds a row) as bf16 rows, through LDS so that neighbouring lanes store neighbouring pieces
template <int D, int CB>
__device__ __forceinline__ void store_rows_at(uint8_t *stage, const f32x16 (&acc)[CB], float scale, bf16_t *p, long ld, int dh, const Rows &at, const Group &g) {
    constexpr int RS = 2 * D + 16, LPR = D / 8, RPI = 64 / LPR;
    const int lane = threadIdx.x & 63, half = lane >> 5, l32 = lane & 31;
#pragma unroll
    for (int c = 0; c < CB; ++c)
#pragma unroll
        for (int gq = 0; gq < 4; ++gq) {
            uint2 w;
            w.x = pack_bf16x2(acc[c][4 * gq] * scale, acc[c][4 * gq + 1] * scale);
            w.y = pack_bf16x2(acc[c][4 * gq + 2] * scale, acc[c][4 * gq + 3] * scale);
            *reinterpret_cast<uint2 *>(stage + l32 * RS + (32 * c + 8 * gq + 4 * half) * 2) = w;
        }
    const int r0 = lane / LPR, cb = (lane % LPR) * 8;
    bf16_t *const first = p + at.t * ld;
#pragma unroll
    for (int i = 0; i < 32 / RPI; ++i) {
        const int r = i * RPI + r0;
        const uint4 v = *reinterpret_cast<const uint4 *>(stage + r * RS + cb * 2);
        if (r < at.left && cb < dh) *reinterpret_cast<uint4 *>(first + at.offset(g, r, ld, dh) + cb) = v;
    }
}

__device__ __forceinline__ float natural_lse(float m, float l, float sl2) { return (m * sl2 + __builtin_amdgcn_logf(l)) * LN2; }

__device__ __forceinline__ int lower_bound(const int *x, int n, int v, bool upper) {     // entries below v, or up to it
    int lo = 0, hi = n;
    while (lo < hi) {
        const int mid = (lo + hi) >> 1;
        if (x[mid] < v || (upper && x[mid] == v)) lo = mid + 1; else hi = mid;
    }
    return lo;
}
struct KeyTile {
    int key, end;               // keys
    int step, steps;            // first step, how many
};
__device__ __forceinline__ KeyTile find_tile(const CrossArgs &a, int y) {
    KeyTile k;
    const int p = find_segment(a.first_tile, 2 * a.S + 1, y), first = a.cuts[p];
    k.key = first + (y - a.first_tile[p]) * TILE_KEYS;
    k.end = a.cuts[p + 1];
    int begin = 0, end = 0;                            // the runs that see the piece: behind the last that ends in front of it
    if (a.S > 0) {
        begin = a.first_step[lower_bound(a.ne, a.S, first, true)];
        end = a.first_step[lower_bound(a.nb, a.S, first, true)];
    }
    const long n = max(end - begin, 0);
    k.step = begin + (int)(n * blockIdx.y / a.parts);
    k.steps = begin + (int)(n * (blockIdx.y + 1) / a.parts) - k.step;
    k.key = __builtin_amdgcn_readfirstlane(k.key);
    k.end = __builtin_amdgcn_readfirstlane(k.end);
    k.step = __builtin_amdgcn_readfirstlane(k.step);
    k.steps = __builtin_amdgcn_readfirstlane(k.steps);
    return k;
}
__device__ __forceinline__ Rows rows_of(const int4 &e) {
    Rows r;
    r.t = __builtin_amdgcn_readfirstlane(e.x);
    r.j = __builtin_amdgcn_readfirstlane(e.y);
    r.left = __builtin_amdgcn_readfirstlane(e.z);
    return r;
}
template <typename K>
hipError_t set_smem(std::atomic<bool> &done, K kern, int bytes) {
    if (done.load(std::memory_order_acquire)) return hipSuccess;
    const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void *>(kern), hipFuncAttributeMaxDynamicSharedMemorySize, bytes);
    if (e == hipSuccess) done.store(true, std::memory_order_release);
    return e;
}

inline size_t table_bytes(int runs) { return ((size_t)(runs + 1) * sizeof(int) + 255) & ~size_t(255); }

}  // namespace

}  // namespace mmt
