// How calls of cross attention are cut into workgroups: the tables that the kernels look their work up in, and the plans that the host makes of
// the runs (the same from the same arrays, so that the size of a workspace and a call agree).
#include "cross_tiles.h"
#include <algorithm>

namespace mmt {

namespace {

// exclusive sums of the runs' items [S + 1], those of a sequence of runs with the same keys at its first; the first run behind its sequence [S]: one workgroup
__global__ __launch_bounds__(1024) void cross_prefix_kernel(CrossArgs a, int tile_rows, int chunk, int *out) {
    __shared__ int sums[16];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int base = 0;
    for (int s0 = 0; s0 < a.S; s0 += 1024) {
        const int s = s0 + threadIdx.x;
        const bool first = first_of_sequence(a, s);
        const int end = behind_sequence(a, s, first);
        const int n = s < a.S && first ? items_of(a.cu[end] - a.cu[s], a.end[s] - a.begin[s], a.nh / a.nkv, tile_rows, chunk) : 0;
        if (s < a.S) out[a.S + 1 + s] = end;
        int sum = n;
#pragma unroll
        for (int o = 1; o < 64; o *= 2) {
            const int v = __shfl_up(sum, o, 64);
            if (lane >= o) sum += v;
        }
        __syncthreads();
        if (lane == 63) sums[wave] = sum;
        __syncthreads();
        int before = base, all = base;
        for (int w = 0; w < 16; ++w) {
            if (w < wave) before += sums[w];
            all += sums[w];
        }
        if (s < a.S) out[s] = before + sum - n;
        base = all;
    }
    if (threadIdx.x == 0) out[a.S] = base;
}

size_t aligned(size_t n) { return (n + 255) & ~size_t(255); }
// runs that follow one another and see the same keys, from s on: the first behind them.  The kernels work on them as on one: 16 continuations of a token each, four
// to a prompt of 6400 keys, 16 heads of 64: 64 us one by one, 43 as four
int behind(const CrossShape &c, int s) {
    int e = s + 1;
    while (e < c.S && e % 64 && c.begin[e] == c.begin[s] && c.end[e] == c.end[s]) ++e;
    return e;
}
// f(first token, first behind, keys) for each such sequence
template <typename F>
void each_sequence(const CrossShape &c, F f) {
    for (int s = 0, e; s < c.S; s = e) {
        e = behind(c, s);
        f(c.cu[s], c.cu[e], c.end[s] - c.begin[s]);
    }
}

void order_runs(const CrossShape &c, CrossArgs &a) {
    if (c.S > 64) return;
    for (int s = 0; s < c.S; s = behind(c, s)) a.order[a.n_sequences++] = (uint8_t)s;
    // (their numbers settle the order of equal ones: a sort that keeps it by itself asks the heap for a buffer)
    std::sort(a.order, a.order + a.n_sequences, [&](uint8_t x, uint8_t y) {
        const int n = c.end[x] - c.begin[x], m = c.end[y] - c.begin[y];
        return n != m ? n > m : x < y;
    });
    for (int i = 0; i < a.n_sequences; ++i) a.last[i] = (uint8_t)(behind(c, a.order[i]) - 1);
}

int items(const CrossShape &c, int rows, int chunk) {
    int n = 0;
    each_sequence(c, [&](int c0, int c1, int keys) { n += items_of(c1 - c0, keys, c.nh / c.nkv, rows, chunk); });
    return n;
}
size_t part_bytes(const CrossShape &c) { return (size_t)c.Tk * 2 * c.nkv * c.d * sizeof(float); }

}  // namespace

// How a forward pass is cut: by the rows of the runs and the keys they see
CrossPlan cross_fwd_plan(int dtype, const CrossShape &c) {
    const int group = c.nh / c.nkv;
    auto count = [&](int rows, int chunk) { return (long)items(c, rows, chunk); };
    // steps of 32 rows and 32 keys
    long few = 0, many = 0, longest = 0;
    each_sequence(c, [&](int c0, int c1, int n_keys) {
        const long keys = (n_keys + 31) / 32, rows = (long)(c1 - c0) * group;
        few += (rows + 31) / 32 * keys;
        many += (rows + 127) / 128 * 4 * keys;
        longest = std::max(longest, keys);
    });
    CrossPlan p = {};
    // Workgroups of 128 rows, two of which share a compute unit and cover each other's beginnings and ends, or of 256, which read keys half as often: where
    // a tile walks 64 steps of 64 keys and more on average.  us, 128 / 256 rows, heads of 128: 4096 tokens of 32 heads on 8 in one run of 8192 keys 524 / 492,
    // of 32 heads in four runs of 2304 175 / 184; of 80, 8 runs of 1024 38 / 42; of 64, 16 runs of 576 34 / 42.
    // Tiles of 32 rows where those of 128 would be less than a third full (us, 128 / 32 rows, 60 runs of 1152 keys, 32 heads of 128, 20 rows each 201 / 196, 45 rows 209 / 231; of 64
    // 130 keys 19 / 15, 21 / 20) or too few.
    const long of128 = count(128, 0);
    p.rows = dtype == DT_F32 ? 16 : many > 3 * few || of128 * c.nkv < 128 ? FEW_ROWS : c.d > 64 && many >= 512 * of128 ? 256 : 128;
    // Long walks of few rows are cut so that there are no more workgroups than fit on the chip at once (bf16: one per compute unit; where two rounds are needed anyway,
    // two).  us, at most 256 / 512 / 1024 workgroups, one token a run: 16 runs of 6144 keys, 8 heads of 128 85 / 84 / 91; 5 of 4000 21 / 25 / 29; 48 that see 5000 keys,
    // four in a row the same 60 / 62 / 70.  A chunk has 8 blocks of 32 keys at least (fp32: 4): one run of 4 heads of 128, 1152 keys, uncut / 16 / 8 / 4 blocks
    // 13.1 / 12.7 / 11.2 / 10.7, 4600 keys 34.7 / 13.5 / 12.5 / 13.2; fp32, heads of 80, 1152 keys 26.6 / 19.0 / 13.7 / 12.3.  Shorter walks stay whole (uncut / cut: 1152
    // keys of 64-wide heads 8.2 / 11.0, of 128 13.2 / 12.0).
    const bool f32 = dtype == DT_F32;
    const long uncut = (p.rows == 128 ? of128 : count(p.rows, 0)) * c.nkv;
    if (p.rows <= FEW_ROWS && uncut < 512 && longest > (f32 ? 12 : c.d <= 64 ? 64 : 32)) {
        const long most = f32 ? 1024 : uncut < 192 ? 256 : 512, want = std::max(few * c.nkv / most, f32 ? 4l : 8l);
        p.chunk = (int)std::min((want + 3) / 4 * 128, 1l << 20);
        while (p.chunk < longest * 32 && count(p.rows, p.chunk) * c.nkv > most) p.chunk += std::max(p.chunk / 16 / 128 * 128, 128);
        if (p.chunk >= longest * 32) p.chunk = 0;
    }
    p.items = (int)(p.chunk ? count(p.rows, p.chunk) : uncut / c.nkv);
    p.table = c.S > 64;
    // Wavefronts share a walk as far as the chip holds all workgroups at once: 256 of eight (wide heads four), 512 of two with wide heads and 1280 with 64-wide ones; beyond those
    // one, or two again where wide heads walk twelve blocks of 32 keys and more on average.  us, 2 / 1, S 60, n 260 / 390 / 577 / 1500: 32 heads of 80 44 / 46, 60 / 64, 89 / 96,
    // 219 / 228, of 128 48 / 44, 75 / 73, 106 / 105, 258 / 258; with 640 workgroups one is faster, S 20, 32 of 80 20 / 18, 26 / 24, 34 / 33, 81 / 85, of 128 24 / 19, 28 / 25, 38 / 33,
    // 107 / 92.  us, most / 2 / 1, S runs of three tokens, n keys each, heads: S 20, 8 heads of 128, n 260 10.5 / 11.1 / 16; S 20, 32 of 128, n 20 15 / 11 / 7, n 577 41 / 36 / 41;
    // S 60, 32 of 128, n 130 48 / 35 / 29, n 577 103 / 98 / 98; S 20, 32 of 64, n 260 18 / 12 / 13; S 60, 32 of 64, n 20 30 / 10 / 8, n 577 67 / 55 / 56.
    const long all = p.items * (long)c.nkv;
    p.waves = all <= 256 || p.chunk ? (c.d <= 64 ? 8 : 4) : c.d <= 64 ? (all <= 1280 ? 2 : 1) : all <= 512 || few >= 12 * uncut / c.nkv ? 2 : 1;
    return p;
}

// [table of items] [parts] [their maxima and sums]
size_t cross_fwd_bytes(const CrossShape &c, const CrossPlan &p) {
    return (p.table ? table_bytes(c.S) : 0) + (p.chunk ? (size_t)p.items * c.nkv * p.rows * (c.d * sizeof(float) + sizeof(float2)) : 0);
}

hipError_t cross_fwd(int dtype, const CrossArgs &args, const CrossShape &c, const CrossPlan &p, void *ws, hipStream_t st) {
    CrossArgs a = args;
    order_runs(c, a);
    uint8_t *at = (uint8_t *)ws;
    if (p.table) {
        a.prefix = (int *)at;
        cross_prefix_kernel<<<1, 1024, 0, st>>>(a, p.rows, p.chunk, (int *)at);
        at += table_bytes(a.S);
    }
    a.chunk = p.chunk;
    if (p.chunk) {
        a.part = (float *)at;
        a.part_ml = (float2 *)(a.part + (size_t)p.items * a.nkv * p.rows * a.d);
    }
    return dtype == DT_F32 ? cross_f32_fwd(a, p, st) : cross_mfma_fwd(a, p, st);
}

// Keys between two places where a run's range begins or ends: steps of the rows that see them, tiles of keys
struct Piece { long steps, tiles; };
constexpr int MOST_PIECES = 1024;      // (a call with more tiles than this has workgroups enough)

// How many workgroups share a tile's rows.  `slots` workgroups run at a time, those with the most steps first: they take at least as long as the k-th round's
// longest k times over, or all steps spread evenly.  A step takes about 2 us (64-wide heads 1.4), a workgroup's beginning and end 5, and what several share
// is written and read once more.  us, 1 / 2 / 4 / 8 parts, the whole backward pass: 4096 tokens of 16 heads of 128 in a run of 700 keys 140 / 107 / 119 / 129,
// 4000 tokens of 16 heads of 64, on 4 in five runs that see 2000 keys 357 / 206 / 134 / 102, 4096 of 64 heads of 128, on 8 in eight runs of 625 309 / 333 / 346 / 407.
int dkv_parts(const CrossShape &c, Piece *pieces, int n_pieces, long tiles) {
    const long slots = c.d > 64 ? 256 : 512, all = tiles * c.nkv;
    if (all == 0 || all >= 2 * slots) return 1;
    std::sort(pieces, pieces + n_pieces, [](const Piece &x, const Piece &y) { return x.steps > y.steps; });
    double work = 0;
    for (int i = 0; i < n_pieces; ++i) work += (double)pieces[i].steps * pieces[i].tiles;
    const double step_us = c.d > 64 ? 2. : 1.4;
    double best = 0;
    int parts = 1;
    for (int n = 1; n <= 16 && (n == 1 || part_bytes(c) * n <= size_t(96) << 20); ++n) {
        const long rounds = (all * n + slots - 1) / slots;
        double steps = work * c.nkv / slots;
        int at = 0;
        long before = 0;                                 // tiles of the pieces in front
        for (long k = 0; k < rounds; ++k) {
            while (at + 1 < n_pieces && (before + pieces[at].tiles) * c.nkv * n <= k * slots) before += pieces[at++].tiles;
            steps = std::max(steps, (double)((k + 1) * ((pieces[at].steps + n - 1) / n)));
        }
        const double us = steps * step_us + rounds * 5 + (n > 1 ? 4 + n * (double)part_bytes(c) / 3e6 : 0);
        if (n == 1 || us < best) { best = us; parts = n; }
    }
    return parts;
}

CrossBwdPlan cross_bwd_plan(int dtype, const CrossShape &c, bool dkv) {
    const int group = c.nh / c.nkv;
    CrossBwdPlan p = {};
    p.rows = dtype == DT_F32 ? 16 : 128;
    // dQ of many short runs: tiles of 32 rows where those of 128 would be less than a third full and there are two rounds of them.  us, 128 / 32 rows, the whole backward pass,
    // 60 runs of 32 heads of 128, 20 keys each: 5 tokens each 58 / 48, 20 tokens 59 / 50, 45 tokens 69 / 66, 90 tokens 96 / 102; 577 keys, 20 tokens 363 / 359; eight runs 14 / 13, 577 keys 62 / 62.
    const long of128 = dtype == DT_F32 ? 0 : items(c, 128, 0);
    if (of128 * c.nkv >= 512 && of128 * 4 > items(c, FEW_ROWS, 0) * 3l) p.rows = FEW_ROWS;
    // Keys are cut into chunks where tiles of rows leave the chip empty and some walk 12 steps of 64 keys and more; a chunk has four steps at least (fp32: two).
    // us, uncut / cut, the whole backward pass, one run of 8 heads of 128: 100 tokens, 768 keys 35 / 28, 2304 keys 78 / 30; 1500 tokens, 768 keys 51 / 54, 2304 keys
    // 109 / 88; fp32, heads of 64, 100 tokens, 2304 keys 76 / 59.
    long walk = 0, longest = 0;
    each_sequence(c, [&](int c0, int c1, int n_keys) {
        const int n = items_of(c1 - c0, 0, group, p.rows, 0);
        const long keys = (n_keys + 63) / 64;
        p.items += n;
        walk += n * keys;
        if (n) longest = std::max(longest, keys);
    });
    if ((long)p.items * c.nkv < 256 && longest >= 12) {
        const long want = std::max(walk * c.nkv / 512, dtype == DT_F32 ? 2l : 4l);
        if (want < longest) {
            p.chunk = (int)want * 64;
            p.items = items(c, p.rows, p.chunk);
        }
    }
    p.table = c.S > 64;
    p.dkv = dkv;
    p.parts = 1;
    if (!dkv) return p;
    // the pieces of the keys: beginnings and ends of the runs that see something, merged
    long tiles = 0, steps = 0, open = 0;                 // steps of all runs, of those that see a piece
    long open16 = 0, walk16 = 0;                         // blocks of 16 rows of the runs that see a piece; that all tiles walk
    Piece pieces[MOST_PIECES];
    int n_pieces = 0;
    int at = 0;
    auto blocks_of = [&](int s, int rows) { return ((long)(c.cu[behind(c, s)] - c.cu[s]) * group + rows - 1) / rows; };
    auto cut = [&](int place) {
        const long n = (place - at + TILE_KEYS - 1) / TILE_KEYS;
        tiles += n;
        walk16 += n * open16;
        if (n && tiles < MOST_PIECES) pieces[n_pieces++] = {open, n};
        at = place;
    };
    int b = 0, e = 0;
    auto next = [&](int s) { while (s < c.S && c.begin[s] == c.end[s]) s = behind(c, s); return s; };
    for (b = next(0), e = b; e < c.S;) {
        if (b < c.S && c.begin[b] <= c.end[e]) {
            cut(c.begin[b]);
            steps += blocks_of(b, STEP_ROWS);
            open += blocks_of(b, STEP_ROWS);
            open16 += blocks_of(b, 16);
            b = next(behind(c, b));
        } else {
            cut(c.end[e]);
            open -= blocks_of(e, STEP_ROWS);
            open16 -= blocks_of(e, 16);
            e = next(behind(c, e));
        }
    }
    cut(c.Tk);
    p.tiles = (int)tiles;
    p.steps = (int)steps;
    if (dtype == DT_F32) {
        // A workgroup for each 16 keys, or, where the keys are many and there are few rows to share out, a wavefront.  us, workgroup / wavefront, the whole backward
        // pass, heads of 64: 400 tokens of 16 heads in 40 runs of 200 keys 122 / 71, of 4 heads in 40 of 75 28 / 21; 1000 of 16 heads in eight runs of 1000 keys 252 / 205;
        // 60 of 4 heads in twelve runs of 83 keys 16.5 / 16.0; 549 in twelve of 168 27 / 29; heads of 80: 1031 tokens of 16 heads in five runs of 420 keys 121 / 130, 1000 in one of
        // 8000 keys 1565 / 1673.
        p.own = tiles * (TILE_KEYS / 16) * c.nkv >= 512 && walk16 <= 8 * tiles;
        // Few keys and many rows: several workgroups share the rows (us, one / several, the whole backward pass: 491 tokens of 64 heads of 80, on 8 in two runs that see 78 keys
        // 197 / 78, 1000 of 16 heads of 64 in one run of 64 keys 53 / 43; from 256 workgroups on 500 keys, 8 heads 57 / 58, 2000 keys, 4 heads 108 / 120).
        const long all = tiles * (TILE_KEYS / 16) * c.nkv;
        while (all < 256 && p.parts < 16 && all * p.parts * 2 <= 1024 && walk16 >= 32 * tiles * p.parts && part_bytes(c) * p.parts * 2 <= size_t(96) << 20) p.parts *= 2;
        return p;
    }
    p.parts = dkv_parts(c, pieces, n_pieces, tiles);
    return p;
}

size_t plan_bytes(int runs) { return runs > PLAN_LDS_RUNS ? aligned((size_t)PLAN_INTS(runs) * sizeof(int)) : 0; }

// [D] [table of items] [tiles] [steps] [what they are made of] [parts: of dQ, then of dK and dV]
size_t cross_bwd_bytes(const CrossShape &c, const CrossBwdPlan &p) {
    size_t n = aligned((size_t)c.Tq * c.nh * sizeof(float)) + (p.table ? table_bytes(c.S) : 0);
    if (p.dkv) n += aligned((size_t)p.tiles * sizeof(int4)) + aligned((size_t)p.steps * sizeof(int4)) + plan_bytes(c.S);
    return n + std::max(p.dkv && p.parts > 1 ? p.parts * part_bytes(c) : 0, p.chunk ? (size_t)p.items * c.nkv * p.rows * c.d * sizeof(float) : 0);
}

hipError_t cross_bwd(int dtype, const CrossArgs &args, const CrossShape &c, const CrossBwdPlan &plan, void *ws, hipStream_t st) {
    CrossArgs a = args;
    CrossBwdPlan p = plan;
    if (!a.dq && p.chunk) { p.chunk = 0; p.items = items(c, p.rows, 0); }
    order_runs(c, a);
    uint8_t *at = (uint8_t *)ws;
    auto take = [&](size_t n) { void *q = at; at += n; return q; };
    a.D = (float *)take(aligned((size_t)a.Tq * a.nh * sizeof(float)));
    a.parts = p.parts;
    a.chunk = p.chunk;
    if (p.table) {
        a.prefix = (int *)take(table_bytes(a.S));
        if (p.items) cross_prefix_kernel<<<1, 1024, 0, st>>>(a, p.rows, p.chunk, const_cast<int *>(a.prefix));
    }
    if (p.dkv && p.tiles) {
        a.tiles = (int4 *)take(aligned((size_t)p.tiles * sizeof(int4)));
        a.steps = (int4 *)take(aligned((size_t)p.steps * sizeof(int4)));
        a.plan = (int *)take(plan_bytes(a.S));
        a.n_tiles = p.tiles; a.n_steps = p.steps;
    }
    a.part = a.dkv_part = (float *)at;                   // one after the other
    if (!p.items && !(p.dkv && p.tiles)) return hipSuccess;
    return dtype == DT_F32 ? cross_f32_bwd(a, p, st) : cross_mfma_bwd(a, p, st);
}

}  // namespace mmt
