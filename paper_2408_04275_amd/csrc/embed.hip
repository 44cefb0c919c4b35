// Embedding of a pack, and its gradient by sorted tokens.
//
// Forward moves each row once.  Backward sorts the tokens by the row that they name, equal ones in their order in the pack, and adds up
// neighbours: a workgroup has a chunk of the order, writes the rows whose tokens it has all of, and leaves partial sums of the (at most two) that
// reach into other chunks for the next launch.  Rows that nobody names are cleared beside it, found absent by a search in the order.
// All of it is bound by memory.  8192 tokens, 4096 wide, 4608 of them encoder features: forward 24 us (4.9 TB/s); back into the fp32 gradient of a table of 32768 rows
// 52 us, the order 11, the sums 36 (4.6 TB/s), the join 5; 16411 tokens, 8192 wide, and a whole bf16 gradient of 131072 rows 493 us, the sums 470 (5.3 TB/s, most of it zeros).
#include "ops.h"
#include "vec8.h"
#include <algorithm>
#include <atomic>

namespace mmt {
namespace {

// where a token's row comes from: row of the table, vocab + row of features, or vocab + features for none
__device__ __forceinline__ int source_of(const EmbedArgs &a, int id) {
    if (id >= 0) return id < a.vocab ? id : a.vocab + a.features;
    return id >= -a.features ? a.vocab - 1 - id : a.vocab + a.features;
}

template <typename T>
__global__ __launch_bounds__(256) void embed_fwd_kernel(EmbedArgs a) {
    const int chunks = a.H / 8;
    const long i = ((long)blockIdx.y * gridDim.x + blockIdx.x) * 256 + threadIdx.x;
    if (i >= (long)a.T * chunks) return;
    const int t = (int)(i / chunks), c = (int)(i % chunks), src = source_of(a, a.ids[t]);
    float v[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    if (src < a.vocab + a.features) {
        const bool text = src < a.vocab;
        load8((text ? (const T *)a.table + (long)src * a.H : (const T *)a.rows + (long)(src - a.vocab) * a.H) + 8 * c, v);
        if (text) {
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] *= a.scale;
        }
    }
    store8((T *)a.y + (long)t * a.H + 8 * c, v);
}

// ---- the order --------------------------------------------------------------------------------------------------------------
// Short packs: each token's place is the number of tokens in front of it, counted: 16 tokens a workgroup, whose threads compare every other token
// with all of them.  One launch, 2 T^2 / 64 vector instructions.
constexpr int RANK_TOKENS = 16, RANK_LOADS = 8;
__global__ __launch_bounds__(256) void embed_rank_kernel(EmbedArgs a, int *order, int *key) {
    __shared__ int counts[RANK_TOKENS][256 + 4];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), t0 = blockIdx.x * RANK_TOKENS, none = a.vocab + a.features;
    const int mine = t0 + (lane & 15) < a.T ? source_of(a, a.ids[t0 + (lane & 15)]) : none;
    int key_of[RANK_TOKENS], count[RANK_TOKENS];
#pragma unroll
    for (int i = 0; i < RANK_TOKENS; ++i) {
        key_of[i] = __builtin_amdgcn_readlane(mine, i);
        count[i] = 0;
    }
    // eight loads on their way: one at a time the kernel waits for memory (the whole backward pass of 4096 tokens, 1024 wide, added to an fp32 gradient 19.9 us, 18.7 so)
    for (int first = 64 * wave; first < a.T; first += 256 * RANK_LOADS) {
        int other[RANK_LOADS];
#pragma unroll
        for (int b = 0; b < RANK_LOADS; ++b) {
            const int u = first + 256 * b + lane;
            other[b] = u < a.T ? a.ids[u] : 0;
        }
#pragma unroll
        for (int b = 0; b < RANK_LOADS; ++b) {
            const int u0 = first + 256 * b, u = u0 + lane;
            const int k = u < a.T ? source_of(a, other[b]) : none + 1;       // behind all
            if (u0 + 64 <= t0) {
#pragma unroll
                for (int i = 0; i < RANK_TOKENS; ++i) count[i] += k <= key_of[i];
            } else if (u0 >= t0 + RANK_TOKENS) {
#pragma unroll
                for (int i = 0; i < RANK_TOKENS; ++i) count[i] += k < key_of[i];
            } else {
#pragma unroll
                for (int i = 0; i < RANK_TOKENS; ++i) count[i] += k < key_of[i] || (k == key_of[i] && u < t0 + i);
            }
        }
    }
#pragma unroll
    for (int i = 0; i < RANK_TOKENS; ++i) counts[i][threadIdx.x] = count[i];
    __syncthreads();
    const int i = threadIdx.x >> 4, x = threadIdx.x & 15;                    // 16 threads a token
    int at = 0;
#pragma unroll
    for (int j = 0; j < 16; ++j) at += counts[i][16 * j + x];
#pragma unroll
    for (int o = 1; o < 16; o *= 2) at += __shfl_xor(at, o, 64);
    const int t = t0 + i;
    if (x == 0 && t < a.T) {
        order[at] = t;
        key[at] = source_of(a, a.ids[t]);
    }
}

// Longer ones: blocks of 512 tokens are put in order by themselves (halves by counting, then by a search in the other half), and a token's
// place is then what a search in every other block says is in front of it; equal ones count in the blocks before its own.  A workgroup of the second
// launch has 64 tokens of a block and all keys in LDS, and each of its wavefronts searches some of the blocks, four at a time.
constexpr int SORT_BLOCK = 512;
typedef __attribute__((address_space(3))) void lds_void;
// entries of N sorted ones (a power of two) that are below v
template <int N>
__device__ __forceinline__ int entries_below(const int *x, int v) {
    int lo = 0;
#pragma unroll
    for (int step = N / 2; step > 0; step /= 2) lo += x[lo + step - 1] < v ? step : 0;
    return lo + (x[lo] < v);
}
__global__ __launch_bounds__(SORT_BLOCK) void embed_blocks_kernel(EmbedArgs a, int *order, int *key) {
    __shared__ __attribute__((aligned(16))) int keys[SORT_BLOCK], sorted[SORT_BLOCK];
    const int i = threadIdx.x, t = blockIdx.x * SORT_BLOCK + i, wave = __builtin_amdgcn_readfirstlane(i >> 6), none = a.vocab + a.features;
    const int mine = t < a.T ? source_of(a, a.ids[t]) : none + 1;            // behind all
    keys[i] = mine;
    __syncthreads();
    const int half = wave / 4 * 256;
    int at = 0;
    auto count = [&](int first, auto f) {
#pragma unroll 4
        for (int j = first; j < first + 64; j += 4) {
            const int4 k = *reinterpret_cast<const int4 *>(keys + j);
            at += f(k.x, j) + f(k.y, j + 1) + f(k.z, j + 2) + f(k.w, j + 3);
        }
    };
    for (int w = 0; w < 4; ++w) {
        if (w < (wave & 3)) count(half + 64 * w, [&](int k, int) { return (int)(k <= mine); });
        else if (w > (wave & 3)) count(half + 64 * w, [&](int k, int) { return (int)(k < mine); });
        else count(half + 64 * w, [&](int k, int j) { return (int)(k < mine || (k == mine && j < i)); });
    }
    sorted[half + at] = mine;
    __syncthreads();
    at += entries_below<256>(sorted + (256 - half), mine + (half > 0));
    key[blockIdx.x * SORT_BLOCK + at] = mine;
    order[blockIdx.x * SORT_BLOCK + at] = t;
}
__global__ __launch_bounds__(256) void embed_merge_kernel(EmbedArgs a, const int *block_order, const int *block_key, int *order, int *key) {
    extern __shared__ __attribute__((aligned(16))) int keys[];               // [blocks][512], then [4][64] counts
    const int blocks = (a.T + SORT_BLOCK - 1) / SORT_BLOCK;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), own = blockIdx.x / (SORT_BLOCK / 64);
    const __amdgpu_buffer_rsrc_t rs = __builtin_amdgcn_make_buffer_rsrc(const_cast<int *>(block_key), 0, blocks * SORT_BLOCK * 4, 0x00020000);
    for (int i = wave; i < blocks * (SORT_BLOCK / 256); i += 4)              // 256 keys each
        __builtin_amdgcn_raw_ptr_buffer_load_lds(rs, (lds_void *)(keys + i * 256), 16, i * 1024 + lane * 16, 0, 0, 0);
    int *const counts = keys + blocks * SORT_BLOCK;
    const int at = blockIdx.x * 64 + lane;
    const int t = block_order[at], mine = block_key[at];
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
    int before = 0;
    for (int b0 = wave; b0 < blocks; b0 += 16) {
        int lo[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) lo[i] = 0;
#pragma unroll
        for (int step = SORT_BLOCK / 2; step > 0; step /= 2)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int b = min(b0 + 4 * i, blocks - 1);
                lo[i] += keys[b * SORT_BLOCK + lo[i] + step - 1] < mine + (b < own) ? step : 0;
            }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int b = min(b0 + 4 * i, blocks - 1);
            const int n = lo[i] + (keys[b * SORT_BLOCK + lo[i]] < mine + (b < own));
            before += b0 + 4 * i < blocks && b != own ? n : 0;
        }
    }
    counts[wave * 64 + lane] = before;
    __syncthreads();
    if (wave == 0 && t < a.T) {
        const int place = counts[lane] + counts[64 + lane] + counts[128 + lane] + counts[192 + lane] + at % SORT_BLOCK;
        order[place] = t;
        key[place] = mine;
    }
}

// Long packs: a radix sort from the lowest eight bits up.  A workgroup has 4096 entries, a wavefront 1024 of them in a row.
constexpr int RADIX_BLOCK = 4096, RADIX_ROUNDS = 16;
struct RadixPass {
    const int *key_in, *order_in;   // null: the ids themselves
    int *key_out, *order_out;
    int *hist;                      // [256][blocks]
    int blocks, shift;
};
__device__ __forceinline__ int radix_key(const EmbedArgs &a, const RadixPass &p, int i) { return p.key_in ? p.key_in[i] : source_of(a, a.ids[i]); }
// lanes of the wavefront whose digit is this lane's (of those that have one)
__device__ __forceinline__ unsigned long long same_digit(int digit, bool live) {
    unsigned long long m = __builtin_amdgcn_ballot_w64(live);
#pragma unroll
    for (int b = 0; b < 8; ++b) {
        const bool bit = (digit >> b) & 1;
        const unsigned long long on = __builtin_amdgcn_ballot_w64(bit);
        m &= bit ? on : ~on;
    }
    return m;
}
__global__ __launch_bounds__(256) void embed_radix_count_kernel(EmbedArgs a, RadixPass p) {
    __shared__ int n[256];
    n[threadIdx.x] = 0;
    __syncthreads();
    const long first = (long)blockIdx.x * RADIX_BLOCK;
    for (int r = 0; r < RADIX_ROUNDS; ++r) {
        const long i = first + r * 256 + threadIdx.x;
        if (i < a.T) atomicAdd(&n[radix_key(a, p, (int)i) >> p.shift & 255], 1);
    }
    __syncthreads();
    p.hist[(size_t)threadIdx.x * p.blocks + blockIdx.x] = n[threadIdx.x];
}
// exclusive sums of hist, in place: one workgroup
__global__ __launch_bounds__(1024) void embed_radix_scan_kernel(RadixPass p) {
    __shared__ int sums[16];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const long all = 256l * p.blocks;
    int base = 0;
    for (long i0 = 0; i0 < all; i0 += 4096) {
        const long i = i0 + threadIdx.x * 4;
        int v[4], n = 0;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            v[e] = i + e < all ? p.hist[i + e] : 0;
            n += v[e];
        }
        int sum = n;
#pragma unroll
        for (int o = 1; o < 64; o *= 2) {
            const int u = __shfl_up(sum, o, 64);
            if (lane >= o) sum += u;
        }
        __syncthreads();
        if (lane == 63) sums[wave] = sum;
        __syncthreads();
        int at = base + sum - n;
        for (int w = 0; w < 16; ++w) {
            if (w < wave) at += sums[w];
            base += sums[w];
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            if (i + e < all) p.hist[i + e] = at;
            at += v[e];
        }
    }
}
__global__ __launch_bounds__(256) void embed_radix_move_kernel(EmbedArgs a, RadixPass p) {
    __shared__ int place[4][256];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const long first = (long)blockIdx.x * RADIX_BLOCK + wave * (64 * RADIX_ROUNDS);
    volatile int *const mine = place[wave];
    for (int d = lane; d < 256; d += 64) mine[d] = 0;
    __builtin_amdgcn_wave_barrier();
    int key[RADIX_ROUNDS];
#pragma unroll
    for (int r = 0; r < RADIX_ROUNDS; ++r) {
        const long i = first + r * 64 + lane;
        key[r] = i < a.T ? radix_key(a, p, (int)i) : 0;
    }
#pragma unroll
    for (int r = 0; r < RADIX_ROUNDS; ++r) {
        const bool live = first + r * 64 + lane < a.T;
        const int d = key[r] >> p.shift & 255;
        const unsigned long long m = same_digit(d, live);
        const bool leads = live && __builtin_amdgcn_mbcnt_hi((uint32_t)(m >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)m, 0)) == 0;
        if (leads) mine[d] = mine[d] + __popcll(m);
        __builtin_amdgcn_wave_barrier();
    }
    __syncthreads();
    {
        int at = p.hist[(size_t)threadIdx.x * p.blocks + blockIdx.x];
        for (int w = 0; w < 4; ++w) {
            const int n = place[w][threadIdx.x];
            place[w][threadIdx.x] = at;
            at += n;
        }
    }
    __syncthreads();
#pragma unroll
    for (int r = 0; r < RADIX_ROUNDS; ++r) {
        const long i = first + r * 64 + lane;
        const bool live = i < a.T;
        const int d = key[r] >> p.shift & 255;
        const unsigned long long m = same_digit(d, live);
        const int before = __builtin_amdgcn_mbcnt_hi((uint32_t)(m >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)m, 0));
        const int start = mine[d];
        __builtin_amdgcn_wave_barrier();
        if (live && before == 0) mine[d] = start + __popcll(m);
        __builtin_amdgcn_wave_barrier();
        if (live) {
            p.key_out[start + before] = key[r];
            p.order_out[start + before] = p.order_in ? p.order_in[i] : (int)i;
        }
    }
}

// ---- the sums -------------------------------------------------------------------------------------------------------------------
struct EmbedSums {
    const int *order, *key;         // [T]
    float *part;                    // [chunks][2][H]: sums of a chunk's first and last row, where those reach into other chunks
    int chunk, chunks, fill_rows;   // tokens a chunk; rows that a clearing workgroup looks at
    int columns;                    // columns a workgroup
};

template <typename T, typename G>
__device__ __forceinline__ void add_old(const EmbedArgs &a, int row, int c, float (&old)[8]) {
    if (row < a.vocab) load8((const G *)a.d_table + (long)row * a.H + c, old);
}
// a row's sum, complete; old: what the table holds, where it is added to
template <typename T, typename G>
__device__ __forceinline__ void put_row(const EmbedArgs &a, int row, int c, const float (&s)[8], const float (&old)[8]) {
    float v[8];
    if (row >= a.vocab) {
        if (a.d_rows) store8((T *)a.d_rows + (long)(row - a.vocab) * a.H + c, s);
        return;
    }
    if (!a.d_table) return;
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = a.accumulate ? old[e] + s[e] * a.scale : s[e] * a.scale;
    store8((G *)a.d_table + (long)row * a.H + c, v);
}
__device__ __forceinline__ bool is_named(const int *key, int n, int row) {
    int lo = 0, hi = n;
    while (lo < hi) {
        const int mid = (lo + hi) >> 1;
        if (key[mid] < row) lo = mid + 1; else hi = mid;
    }
    return lo < n && key[lo] == row;
}

// Workgroups of the first chunks * (H / columns) have a chunk and some columns each, eight tokens' rows (and the old contents of the rows that
// end among them) on their way at a time; the others clear rows.
constexpr int SUM_ROWS = 8;
template <typename T, typename G>
__global__ __launch_bounds__(256) void embed_sum_kernel(EmbedArgs a, EmbedSums s) {
    const int slabs = (a.H + s.columns - 1) / s.columns, none = a.vocab + a.features;
    const int block = blockIdx.y * gridDim.x + blockIdx.x, chunk = block / slabs;
    if (chunk >= s.chunks) {
        __shared__ int clear[64];
        const int first = (a.accumulate || !a.d_table ? a.vocab : 0) + (block - s.chunks * slabs) * s.fill_rows;
        const int rows = min(s.fill_rows, (a.d_rows ? none : a.vocab) - first);
        if ((int)threadIdx.x < rows) clear[threadIdx.x] = !is_named(s.key, a.T, first + threadIdx.x);
        __syncthreads();
        const u32x4 zero = {0u, 0u, 0u, 0u};
        for (int r = 0; r < rows; ++r) {
            if (!clear[r]) continue;
            const int row = first + r;
            const bool text = row < a.vocab;
            u32x4 *out = text ? (u32x4 *)((G *)a.d_table + (long)row * a.H) : (u32x4 *)((T *)a.d_rows + (long)(row - a.vocab) * a.H);
            for (int i = threadIdx.x; i < a.H * (int)(text ? sizeof(G) : sizeof(T)) / 16; i += blockDim.x) __builtin_nontemporal_store(zero, out + i);
        }
        return;
    }
    const int column = (block % slabs) * s.columns + threadIdx.x * 8;
    const bool live = column < a.H;
    const int c = live ? column : 0;                   // (a wavefront stays whole: its lanes hold the places)
    const int p0 = chunk * s.chunk, p1 = min(p0 + s.chunk, a.T), lane = threadIdx.x & 63;
    float sum[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    bool whole = true;                                 // the present row's first token is in this chunk
    int keys = 0, tokens = 0;                          // lane i: key and token of place base - 1 + i
    int base = p0;
    for (int p = p0; p < p1; p += SUM_ROWS) {
        if (p == p0 || p - base > 62 - SUM_ROWS - 1) {
            base = p;
            const int at = base - 1 + lane;
            keys = at >= 0 && at < a.T ? s.key[at] : -1;
            tokens = at >= 0 && at < a.T ? s.order[at] : 0;
            if (p == p0) whole = __builtin_amdgcn_readlane(keys, 0) != __builtin_amdgcn_readlane(keys, 1);
        }
        int row[SUM_ROWS + 1];
        Raw8<T> x[SUM_ROWS];
        float old[SUM_ROWS][8];
#pragma unroll
        for (int i = 0; i <= SUM_ROWS; ++i) row[i] = __builtin_amdgcn_readlane(keys, p - base + 1 + i);
#pragma unroll
        for (int i = 0; i < SUM_ROWS; ++i)
            if (p + i < p1 && row[i] != none) x[i] = load_plain8((const T *)a.dy + (long)__builtin_amdgcn_readlane(tokens, p - base + 1 + i) * a.H + c);
        if (a.accumulate && a.d_table) {
#pragma unroll
            for (int i = 0; i < SUM_ROWS; ++i)
                if (p + i < p1 && row[i] != row[i + 1] && row[i] != none) add_old<T, G>(a, row[i], c, old[i]);
        }
#pragma unroll
        for (int i = 0; i < SUM_ROWS; ++i) {
            if (p + i >= p1 || row[i] == none) continue;
            float v[8];
            unpack8(x[i], v);
#pragma unroll
            for (int e = 0; e < 8; ++e) sum[e] += v[e];
            const bool ends = row[i] != row[i + 1], last = p + i + 1 == p1;
            if (ends && whole) { if (live) put_row<T, G>(a, row[i], c, sum, old[i]); }
            else if ((ends || last) && live) store8(s.part + ((size_t)chunk * 2 + (whole ? 1 : 0)) * a.H + c, sum);
            if (ends) {
                whole = true;
#pragma unroll
                for (int e = 0; e < 8; ++e) sum[e] = 0.f;
            }
        }
    }
}

// Rows whose tokens stand in several chunks: the workgroup of the chunk that a row begins in adds up the chunks' sums, four threads per eight
// columns, a quarter of the chunks each
constexpr int JOIN_COLUMNS = 512;
template <typename T, typename G>
__global__ __launch_bounds__(256) void embed_join_kernel(EmbedArgs a, EmbedSums s) {
    __shared__ float red[3][64][9];
    const int slabs = (a.H + JOIN_COLUMNS - 1) / JOIN_COLUMNS, chunk = blockIdx.x / slabs;
    const int last = min((chunk + 1) * s.chunk, a.T) - 1;
    if (last + 1 >= a.T) return;
    const int row = s.key[last], next = s.key[last + 1], first = s.key[max(chunk * s.chunk - 1, 0)];
    if (row == a.vocab + a.features || next != row) return;          // ends here
    if (chunk > 0 && first == row) return;                           // began earlier
    int lo = last + 1, hi = a.T;                       // the row's end in the order
    while (lo < hi) {
        const int mid = (lo + hi) >> 1;
        if (s.key[mid] == row) lo = mid + 1; else hi = mid;
    }
    const int n = (lo - 1) / s.chunk - chunk;          // chunks behind this one
    const int c = (blockIdx.x % slabs) * JOIN_COLUMNS + (threadIdx.x & 63) * 8, q = threadIdx.x >> 6;
    const bool live = c < a.H;
    const size_t stride = (size_t)2 * a.H;
    const float *part = s.part + (size_t)(chunk + 1) * stride + c;       // their first rows
    float sum[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f}, old[8];
    if (live) {
        if (q == 0) {
            load8(s.part + (size_t)chunk * stride + a.H + c, sum);
            if (a.accumulate && a.d_table) add_old<T, G>(a, row, c, old);
        }
        int j = q;
        for (; j + 12 < n; j += 16) {
            float v[4][8];
#pragma unroll
            for (int i = 0; i < 4; ++i) load8(part + (size_t)(j + 4 * i) * stride, v[i]);
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int e = 0; e < 8; ++e) sum[e] += v[i][e];
        }
        for (; j < n; j += 4) {
            float v[8];
            load8(part + (size_t)j * stride, v);
#pragma unroll
            for (int e = 0; e < 8; ++e) sum[e] += v[e];
        }
    }
    if (q > 0) {
#pragma unroll
        for (int e = 0; e < 8; ++e) red[q - 1][threadIdx.x & 63][e] = sum[e];
    }
    __syncthreads();
    if (q > 0 || !live) return;
#pragma unroll
    for (int w = 0; w < 3; ++w)
#pragma unroll
        for (int e = 0; e < 8; ++e) sum[e] += red[w][threadIdx.x][e];
    put_row<T, G>(a, row, c, sum, old);
}

// ---- sizes ---------------------------------------------------------------------------------------------------------------------------
constexpr int RANK_MAX = 4096, MERGE_MAX = 32768;      // the longest packs that are ordered by counting, and by blocks (whose keys fill 128 KB of LDS)
// Tokens a chunk: 16, up to 64 while the chip has work enough (fewer rows reach into other chunks, whose partial sums are written and read back), and as
// many as keep the chunks' number within 2048.  Short packs: 8, one round of a workgroup, from two chunks on (us, 16 / 8, fp32 gradient 1024 wide: 9 tokens
// 9.8 / 11.8, 33 14.2 / 11.6, 1000 17.4 / 14.8; 4096 wide, 2000 tokens 21.7 / 21.5, written as bf16 22.1 / 23.0).
int chunk_of(int T, int H) {
    int c = T >= 16 && (long)ceil_div(T, 8) * ceil_div(H, 2048) <= 256 ? 8 : 16;
    while (c < 64 && (long)ceil_div(T, 2 * c) * ceil_div(H, 2048) >= 1024) c *= 2;
    return std::max(c, (T / 2048 + 8) / 8 * 8);
}
size_t aligned(size_t n) { return (n + 255) & ~size_t(255); }
int radix_blocks(int T) { return ceil_div(T, RADIX_BLOCK); }

// a launch holds fewer than 2^32 threads along x
dim3 rows_grid(long blocks) { return dim3((unsigned)std::min(blocks, 1l << 20), (unsigned)((blocks + (1l << 20) - 1) >> 20)); }

template <typename T, typename G>
hipError_t sums(const EmbedArgs &a, const EmbedSums &s, hipStream_t st) {
    const int threads = std::min(256, (a.H / 8 + 63) / 64 * 64), slabs = ceil_div(a.H, s.columns);
    const int first = a.accumulate || !a.d_table ? a.vocab : 0, rows = (a.d_rows ? a.vocab + a.features : a.vocab) - first;
    const int blocks = s.chunks * slabs + ceil_div(rows, s.fill_rows);
    if (blocks) embed_sum_kernel<T, G><<<rows_grid(blocks), threads, 0, st>>>(a, s);
    if (s.chunks > 1) embed_join_kernel<T, G><<<s.chunks * ceil_div(a.H, JOIN_COLUMNS), 256, 0, st>>>(a, s);
    return blocks ? hipGetLastError() : hipSuccess;
}

}  // namespace

hipError_t embed_fwd(int dtype, const EmbedArgs &a, hipStream_t st) {
    if (a.T == 0) return hipSuccess;
    const dim3 grid = rows_grid(((long)a.T * (a.H / 8) + 255) / 256);
    if (dtype == DT_F32) embed_fwd_kernel<float><<<grid, 256, 0, st>>>(a);
    else embed_fwd_kernel<bf16_t><<<grid, 256, 0, st>>>(a);
    return hipGetLastError();
}

// [key] [order] [partial sums], and for longer packs [key] [order] [counts] of the sort
size_t embed_bwd_bytes(int T, int H) {
    const size_t most = (size_t)std::min(ceil_div(T, 8), 2048) * 2 * H * sizeof(float);        // (never falls; longer chunks need less)
    return 2 * aligned((size_t)T * sizeof(int)) + aligned(most) +
           (T > RANK_MAX ? 2 * aligned(((size_t)T + SORT_BLOCK) * sizeof(int)) : 0) + (T > MERGE_MAX ? aligned(256ul * radix_blocks(T) * sizeof(int)) : 0) + 256;
}

hipError_t embed_bwd(int dtype, const EmbedArgs &a, hipStream_t st) {
    EmbedSums s = {};
    uint8_t *at = (uint8_t *)a.ws;
    auto take = [&](size_t n) { void *p = at; at += aligned(n); return p; };
    int *key = (int *)take((size_t)a.T * sizeof(int)), *order = (int *)take((size_t)a.T * sizeof(int));
    int *key2 = nullptr, *order2 = nullptr;
    if (a.T > RANK_MAX) {
        key2 = (int *)take(((size_t)a.T + SORT_BLOCK) * sizeof(int));
        order2 = (int *)take(((size_t)a.T + SORT_BLOCK) * sizeof(int));
    }
    if (a.T > MERGE_MAX) {
        RadixPass p = {};
        p.blocks = radix_blocks(a.T);
        p.hist = (int *)take(256ul * p.blocks * sizeof(int));
        int bits = 1;
        while ((a.vocab + a.features) >> bits) ++bits;
        const int passes = (bits + 7) / 8;
        for (int i = 0; i < passes; ++i) {
            const bool to_first = (passes - i) % 2;    // the last pass writes key and order
            p.key_out = to_first ? key : key2; p.order_out = to_first ? order : order2;
            p.shift = 8 * i;
            embed_radix_count_kernel<<<p.blocks, 256, 0, st>>>(a, p);
            embed_radix_scan_kernel<<<1, 1024, 0, st>>>(p);
            embed_radix_move_kernel<<<p.blocks, 256, 0, st>>>(a, p);
            p.key_in = p.key_out; p.order_in = p.order_out;
        }
    } else if (a.T > RANK_MAX) {
        static std::atomic<bool> done{false};
        const int blocks = ceil_div(a.T, SORT_BLOCK), lds = (blocks * SORT_BLOCK + 256) * (int)sizeof(int);
        if (!done.load(std::memory_order_acquire)) {
            const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void *>(embed_merge_kernel), hipFuncAttributeMaxDynamicSharedMemorySize, (MERGE_MAX + 256) * (int)sizeof(int));
            if (e != hipSuccess) return e;
            done.store(true, std::memory_order_release);
        }
        embed_blocks_kernel<<<blocks, SORT_BLOCK, 0, st>>>(a, order2, key2);
        embed_merge_kernel<<<ceil_div(a.T, 64), 256, lds, st>>>(a, order2, key2, order, key);
    } else if (a.T > 0) embed_rank_kernel<<<ceil_div(a.T, RANK_TOKENS), 256, 0, st>>>(a, order, key);
    s.key = key; s.order = order;
    s.chunk = chunk_of(a.T, a.H);
    s.chunks = ceil_div(a.T, s.chunk);
    s.part = (float *)at;
    s.fill_rows = 16;
    s.columns = std::min(2048, (a.H / 8 + 63) / 64 * 64 * 8);
    if (dtype == DT_F32) return sums<float, float>(a, s, st);
    return a.table_f32 ? sums<bf16_t, float>(a, s, st) : sums<bf16_t, bf16_t>(a, s, st);
}

}  // namespace mmt
