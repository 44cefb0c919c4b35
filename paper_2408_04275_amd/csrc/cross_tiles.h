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

// inclusive sums over the wavefront, in the vector ALU
template <int CTRL, int ROWS> __device__ __forceinline__ int scan_step(int v) { return v + __builtin_amdgcn_update_dpp(0, v, CTRL, ROWS, 0xf, false); }
__device__ __forceinline__ int wave_scan(int v) {
    v = scan_step<0x111, 0xf>(v);           // row_shr 1, 2, 4, 8
    v = scan_step<0x112, 0xf>(v);
    v = scan_step<0x114, 0xf>(v);
    v = scan_step<0x118, 0xf>(v);
    v = scan_step<0x142, 0xa>(v);           // row_bcast 15 to rows 1 and 3
    return scan_step<0x143, 0xc>(v);        // row_bcast 31 to rows 2 and 3
}

struct Item {
    int q0, rows, lo, hi;       // run: first token, rows of a key/value head, keys
    int index, first;           // the item's number within its run; of the run's first item among all
};

// Of the 64 runs from a multiple of 64 on, one per lane: is it the first that sees its keys, and which is the first behind those that see the same
__device__ __forceinline__ bool first_of_sequence(const CrossArgs &a, int s) {
    return (s & 63) == 0 || (s < a.S && (a.begin[s] != a.begin[s - 1] || a.end[s] != a.end[s - 1]));
}
__device__ __forceinline__ int behind_sequence(const CrossArgs &a, int s, bool first) {
    const uint64_t firsts = __builtin_amdgcn_ballot_w64(first), later = firsts & (~0ull << (s & 63)) & ~(1ull << (s & 63));
    return min((s & ~63) + (later ? __builtin_ctzll(later) : 64), a.S);
}

// Item y of all runs' items.  Up to 64 runs: one per lane, those with the most keys first (the workgroups that start last are then the
// shortest), their items added up across the wavefront; more: from the table that cross_prefix_kernel left.
__device__ __forceinline__ Item find_item(const CrossArgs &a, int y, int tile_rows, int chunk) {
    const int group = a.nh / a.nkv, lane = threadIdx.x & 63;
    Item it;
    if (a.S <= 64) {
        int c0 = 0, c1 = 0, lo = 0, hi = 0;
        const int from = a.order[lane] * 4, to = a.last[lane] * 4;       // the lane's place, from the runs of those numbers
        if (lane < a.S) { c0 = a.cu[lane]; c1 = a.cu[lane + 1]; lo = a.begin[lane]; hi = a.end[lane]; }
        c0 = __builtin_amdgcn_ds_bpermute(from, c0);
        c1 = __builtin_amdgcn_ds_bpermute(to, c1);
        lo = __builtin_amdgcn_ds_bpermute(from, lo);
        hi = __builtin_amdgcn_ds_bpermute(from, hi);
        const int n = lane < a.n_sequences ? items_of(c1 - c0, hi - lo, group, tile_rows, chunk) : 0;
        const int sum = wave_scan(n);
        const int s = min(__popcll(__builtin_amdgcn_ballot_w64(sum <= y)), 63);
        it.q0 = __builtin_amdgcn_readlane(c0, s);
        it.rows = (__builtin_amdgcn_readlane(c1, s) - it.q0) * group;
        it.lo = __builtin_amdgcn_readlane(lo, s);
        it.hi = __builtin_amdgcn_readlane(hi, s);
        it.first = __builtin_amdgcn_readlane(sum - n, s);
    } else {
        const int s = __builtin_amdgcn_readfirstlane(find_segment(a.prefix, a.S, y));
        it.q0 = __builtin_amdgcn_readfirstlane(a.cu[s]);
        it.rows = (__builtin_amdgcn_readfirstlane(a.cu[a.prefix[a.S + 1 + s]]) - it.q0) * group;
        it.lo = __builtin_amdgcn_readfirstlane(a.begin[s]);
        it.hi = __builtin_amdgcn_readfirstlane(a.end[s]);
        it.first = __builtin_amdgcn_readfirstlane(a.prefix[s]);
    }
    it.index = y - it.first;
    return it;
}

// Division of a small number (below group + 128) by the group: the high half of a product with ceil(2^31 / group), exact while number * group < 2^31, for
// every group (a case of its own for groups of one becomes a branch at each row)
struct Group {
    int n;
    uint32_t magic;
    __device__ __forceinline__ explicit Group(int n_) : n(n_), magic((0x80000000u + (uint32_t)n_ - 1u) / (uint32_t)n_) {}
    __device__ __forceinline__ explicit Group(const CrossArgs &a) : Group(a.nh / a.nkv) {}
    __device__ __forceinline__ int token(int r) const { return (int)__umulhi((uint32_t)r * 2u, magic); }
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
        const uint32_t there = (at.offset(g, row, ld, dh) + unit * 8) * 2u, off = row < at.left && unit * 8 < dh ? there : 0x80000000u;
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
    const __amdgpu_buffer_rsrc_t rs = __builtin_amdgcn_make_buffer_rsrc(p + at.t * ld, 0, 0x7fff0000, 0x00020000);
    Rows here = at;
    asm volatile("" : "+s"(here.j));                   // (offsets kept from the copies in front of the walk would fill its registers)
    u32x4 v[32 / RPI];
#pragma unroll
    for (int i = 0; i < 32 / RPI; ++i) v[i] = *reinterpret_cast<const u32x4 *>(stage + (i * RPI + r0) * RS + cb * 2);
#pragma unroll
    for (int i = 0; i < 32 / RPI; ++i) {               // (rows that do not exist are behind the buffer's end: a branch each would make every read wait for the store in front)
        const int r = i * RPI + r0;
        const uint32_t off = (here.offset(g, r, ld, dh) + cb) * 2u;
        __builtin_amdgcn_raw_buffer_store_b128(v[i], rs, (int)(r < at.left && cb < dh ? off : 0x80000000u), 0, 0);
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
// ---- dK, dV: what is walked ---------------------------------------------------------------------------------------------------
// The runs that see something begin and end in their order; the others get the last one's beginning and end (nb, ne).  All those places
// together, sorted, cut the keys into pieces (cuts, [2 S + 2]) whose keys are seen by the same runs, and these follow one another.  A tile is up to
// 128 keys of a piece: {key, end of the piece, first step, steps}; a step up to 64 rows of a sequence of runs: {token, head of the group, rows}.
// One workgroup makes both lists; it stands in front of dQ's, which do not need them, but dK/dV's launch waits for it: with several hundred runs it is what dQ's launch takes (32 heads
// of 128, 8 tokens and 64 keys each: 300 runs 164 us, 92 without the lists; 1000 runs 820 and 284).
constexpr int PLAN_LDS_RUNS = 256;      // as many runs' places are kept in LDS while they are searched (more: in the workspace)
constexpr int PLAN_INTS(int runs) { return 4 * (runs + 1) + 2 * (2 * runs + 2); }
constexpr int PLAN_SORTED = 1024;
constexpr int PLAN_LDS = (PLAN_INTS(PLAN_LDS_RUNS) + 32 + PLAN_SORTED) * 4;
template <int THREADS>
__device__ __forceinline__ int block_scan(int v, bool max, int *sums) {      // inclusive
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
    for (int o = 1; o < 64; o *= 2) {
        const int u = __shfl_up(v, o, 64);
        if (lane >= o) v = max ? ::max(v, u) : v + u;
    }
    __syncthreads();
    if (lane == 63) sums[wave] = v;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < THREADS / 64; ++w)
        if (w < wave) v = max ? ::max(v, sums[w]) : v + sums[w];
    return v;
}
template <int THREADS>
__device__ void make_plan(const CrossArgs &a, int *lds) {
    int *const sums = lds, *const carry = lds + 16;
    const int group = a.nh / a.nkv, S = a.S;
    int *const nb = S <= PLAN_LDS_RUNS ? lds + 32 : a.plan, *const ne = nb + S + 1, *const first_step = ne + S + 1, *const behind = first_step + S + 1, *const cuts = behind + S + 1,
        *const first_tile = cuts + 2 * S + 2;
    if (threadIdx.x < 3) carry[threadIdx.x] = 0;
    __syncthreads();
    for (int s0 = 0; s0 < S; s0 += THREADS) {
        const int s = s0 + threadIdx.x;
        int b = 0, e = 0, n = 0;
        const bool first = first_of_sequence(a, s);
        const int end = behind_sequence(a, s, first);
        if (s < S) {
            const int lo = a.begin[s], hi = a.end[s], c0 = a.cu[s], c1 = a.cu[end];
            if (lo < hi) { b = lo; e = hi; n = first ? ((c1 - c0) * group + STEP_ROWS - 1) / STEP_ROWS : 0; }
            behind[s] = end;
        }
        b = max(block_scan<THREADS>(b, true, sums), carry[0]);
        e = max(block_scan<THREADS>(e, true, sums), carry[1]);
        const int sum = block_scan<THREADS>(n, false, sums) + carry[2];
        if (s < S) { nb[s] = b; ne[s] = e; first_step[s] = sum - n; }
        __syncthreads();
        if (threadIdx.x == THREADS - 1) { carry[0] = b; carry[1] = e; carry[2] = sum; }
        __syncthreads();
    }
    const int all = carry[2];
    __syncthreads();
    if (threadIdx.x == 0) { first_step[S] = all; cuts[0] = 0; cuts[2 * S + 1] = a.Tk; carry[0] = 0; }
    __threadfence_block();
    __syncthreads();
    for (int s = threadIdx.x; s < S; s += THREADS) {
        cuts[1 + s + lower_bound(ne, S, nb[s], false)] = nb[s];
        cuts[1 + s + lower_bound(nb, S, ne[s], true)] = ne[s];
    }
    __threadfence_block();
    __syncthreads();
    for (int p0 = 0; p0 < 2 * S + 1; p0 += THREADS) {
        const int p = p0 + threadIdx.x, n = p < 2 * S + 1 ? (cuts[p + 1] - cuts[p] + TILE_KEYS - 1) / TILE_KEYS : 0;
        const int sum = block_scan<THREADS>(n, false, sums) + carry[0];
        if (p < 2 * S + 1) first_tile[p] = sum - n;
        __syncthreads();
        if (threadIdx.x == THREADS - 1) carry[0] = sum;
        __syncthreads();
    }
    __threadfence_block();
    __syncthreads();
    // tiles with the most steps first, as far as LDS holds their numbers: the workgroups that start last are then the shortest
    int *const lengths = lds + 32 + PLAN_INTS(PLAN_LDS_RUNS);
    const bool sorted = a.n_tiles <= PLAN_SORTED;
    auto tile_of = [&](int y) {
        const int p = find_segment(first_tile, 2 * S + 1, y), first = cuts[p];
        // the runs that see the piece: behind the last that ends in front of it
        const int begin = S > 0 ? first_step[lower_bound(ne, S, first, true)] : 0, end = S > 0 ? first_step[lower_bound(nb, S, first, true)] : 0;
        return make_int4(first + (y - first_tile[p]) * TILE_KEYS, cuts[p + 1], begin, max(end - begin, 0));
    };
    for (int y = threadIdx.x; y < a.n_tiles; y += THREADS) {
        const int4 v = tile_of(y);
        if (sorted) lengths[y] = v.w;
        else a.tiles[y] = v;
    }
    if (sorted) {
        __syncthreads();
        for (int y = threadIdx.x; y < a.n_tiles; y += THREADS) {
            const int4 v = tile_of(y);
            int at = 0;
            for (int i = 0; i < a.n_tiles; ++i) at += lengths[i] > v.w || (lengths[i] == v.w && i < y);
            a.tiles[at] = v;
        }
    }
    for (int i = threadIdx.x; i < a.n_steps; i += THREADS) {
        const int s = find_segment(first_step, S, i), row = (i - first_step[s]) * STEP_ROWS, tok = row / group, c0 = a.cu[s];
        a.steps[i] = make_int4(c0 + tok, row - tok * group, min((a.cu[behind[s]] - c0) * group - row, STEP_ROWS), 0);
    }
}

struct KeyTile {
    int key, end;               // keys
    int step, steps;            // first step, how many
};
// Entries of the lists, which an earlier launch has written: scalar loads, which do not queue up behind the copies into LDS (as vector loads they cost dK/dV
// up to a tenth: the compiler waits for every copy in flight)
__device__ __forceinline__ int4 entry_of(const int4 *list, long i) {
    typedef int Four __attribute__((ext_vector_type(4)));
    const Four v = *(const __attribute__((address_space(4))) Four *)(uintptr_t)(list + i);
    return make_int4(v.x, v.y, v.z, v.w);
}
__device__ __forceinline__ KeyTile find_tile(const CrossArgs &a, int y) {
    const int4 v = entry_of(a.tiles, y);
    KeyTile k;
    k.key = v.x;
    k.end = v.y;
    const int begin = v.z;
    const long n = v.w;
    k.step = begin + (int)(n * blockIdx.y / a.parts);
    k.steps = begin + (int)(n * (blockIdx.y + 1) / a.parts) - k.step;
    return k;
}
__device__ __forceinline__ Rows rows_of(const int4 &e) {
    Rows r;
    r.t = e.x; r.j = e.y; r.left = e.z;
    return r;
}
template <typename K>
hipError_t set_smem(std::atomic<bool> &done, K kern, int bytes) {
    if (done.load(std::memory_order_acquire)) return hipSuccess;
    const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void *>(kern), hipFuncAttributeMaxDynamicSharedMemorySize, bytes);
    if (e == hipSuccess) done.store(true, std::memory_order_release);
    return e;
}

// dQ from the sums over chunks of keys: the workgroups of a tile's chunks share out its rows
template <typename T, int ROWS>
__global__ __launch_bounds__(256) void cross_dq_sum_kernel(CrossArgs a) {
    const int head = blockIdx.x % a.nkv, dh = a.d;
    const Item it = find_item(a, blockIdx.x / a.nkv, ROWS, a.chunk);
    const int parts = max((it.hi - it.lo + a.chunk - 1) / a.chunk, 1), mine_of = it.index % parts;
    if (parts == 1) return;
    const Group g(a);
    const Rows mine(it, g, it.index / parts * ROWS);
    const int quads = dh / 4, rows = min(mine.left, ROWS);
    const size_t stride = (size_t)a.nkv * ROWS * dh;
    const float *part = a.part + (size_t)(blockIdx.x - mine_of * a.nkv) * ROWS * dh;
    T *const out = (T *)a.dq + mine.t * a.lddq + (long)head * g.n * dh;
    for (int e = mine_of * 256 + threadIdx.x; e < rows * quads; e += parts * 256) {
        const int r = e / quads, c = e % quads * 4;
        const float *p = part + r * dh + c;
        f32x4 x = {0.f, 0.f, 0.f, 0.f};
        for (int j0 = 0; j0 < parts; j0 += 8) {
            f32x4 y[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) y[i] = j0 + i < parts ? *reinterpret_cast<const f32x4 *>(p + (j0 + i) * stride) : f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int i = 0; i < 8; ++i) x += y[i];
        }
        x *= a.scale;
        T *const to = out + mine.offset(g, r, a.lddq, dh) + c;
        if constexpr (sizeof(T) == 4) *reinterpret_cast<f32x4 *>(to) = x;
        else *reinterpret_cast<uint2 *>(to) = make_uint2(pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3]));
    }
}

// The parts of dK (scaled) and dV, added in order, as bf16 rows; a thread has four features
template <typename T>
__global__ __launch_bounds__(256) void cross_dkv_sum_kernel(CrossArgs a) {
    const int nk = a.nkv * a.d, quads = 2 * nk / 4;
    const long idx = (long)blockIdx.x * 256 + threadIdx.x;
    if (idx >= (long)a.Tk * quads) return;
    const int t = (int)(idx / quads), c = (int)(idx % quads) * 4;
    const size_t stride = (size_t)a.Tk * 2 * nk;
    const float *p = a.dkv_part + (size_t)t * 2 * nk + c;
    f32x4 x = *reinterpret_cast<const f32x4 *>(p);
    for (int i = 1; i < a.parts; ++i) x += *reinterpret_cast<const f32x4 *>(p + i * stride);
    const bool is_k = c < nk;
    if (is_k) x *= a.scale;
    T *out = is_k ? (T *)a.dk + t * a.lddk + c : (T *)a.dv + t * a.lddv + c - nk;
    if constexpr (sizeof(T) == 4) *reinterpret_cast<f32x4 *>(out) = x;
    else *reinterpret_cast<uint2 *>(out) = make_uint2(pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3]));
}

inline size_t table_bytes(int runs) { return ((size_t)(2 * runs + 1) * sizeof(int) + 255) & ~size_t(255); }

}  // namespace

}  // namespace mmt
