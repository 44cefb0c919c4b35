// Pieces that the bf16 attention kernels are made of: 64-row tiles of a row-major tensor in LDS, their copies, fragments and transposed
// fragments, and results on their way out (see attn_mfma.hip for the layout that all of them share).
#pragma once
#include "common.h"
#include <type_traits>

namespace mmt {

namespace {

constexpr float LOG2E = 1.4426950408889634f, LN2 = 0.6931471805599453f;

// Swizzle of the 16-byte units of a tile row in LDS: unit u of row `row` stands at position u ^ swz_unit<D>(row).
// What it has to achieve was measured with a microbenchmark of LDS read patterns: a 16-byte-per-lane read is served
// 16 lanes at a time, lanes 0-7 together with 24-31, 8-15 with 16-23 (and the same in the upper half), an 8-byte
// transposing read 32 lanes at a time, lanes 0-31 and 32-63, each at full rate when its lanes fall into distinct slots modulo 256
// bytes.  A fragment read covers 32 consecutive rows at one unit: rows 0-7 and 24-31 have to differ, and rows 8-23.  A transposing
// read covers, with half a wavefront, four consecutive rows at four consecutive units (8 bytes a lane): the four rows have to differ in
// the unit bits above the lowest two.  With 256-byte rows (D = 128) the row's two lowest bits go there and its next two below them;
// with 128-byte rows (D = 64) the lowest bit is in the address as it is.  (With the lowest bit alone above, half of the lanes of a
// transposing read were served at a time, and LDS was what the dK/dV kernel waited for.)
template <int D>
__device__ __forceinline__ int swz_unit(int row) {
    if constexpr (D == 128) return (row & 2) << 2 | (row & 1) << 2 | (row >> 1 & 2) | (row >> 3 & 1);
    else return (row & 2) << 1 | (row >> 1 & 2) | (row >> 3 & 1);
}

__device__ __forceinline__ bf16x8 pack8(const float *v) {
    bf16x8 r;
#pragma unroll
    for (int i = 0; i < 8; ++i) r[i] = (__bf16)v[i];
    return r;
}

__device__ __forceinline__ f32x16 zero16() {
    f32x16 z;
#pragma unroll
    for (int i = 0; i < 16; ++i) z[i] = 0.f;
    return z;
}

#define MFMA(a, b, c) __builtin_amdgcn_mfma_f32_32x32x16_bf16((a), (b), (c), 0, 0, 0)

typedef __attribute__((address_space(3))) void lds_void;
typedef __attribute__((ext_vector_type(4))) uint32_t rawx4;

__device__ __forceinline__ void lds_barrier() {
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
}

// fragment of a row-major [rows][D] tile (row bytes 2 D): row, k-slice ks (16 features), lane half
template <int D>
__device__ __forceinline__ bf16x8 frag_k(const uint8_t *tile, int row, int ks, int half) {
    constexpr int UPR = D / 8;
    return *reinterpret_cast<const bf16x8 *>(tile + (row * UPR + ((ks * 2 + half) ^ swz_unit<D>(row))) * 16);
}

typedef __attribute__((ext_vector_type(4))) short shortx4;
typedef __attribute__((ext_vector_type(8))) short shortx8;

// One wavefront's share of the copies of [64][D] tiles out of a row-major tensor: N copies of 1 KiB per tile, copy
// (first + i) of a tile covering its rows (first + i) * 512 / D ...  What depends on the lane is computed once
// (init); a copy then costs one addition.  Rows at or beyond the end of the tensor read as zero (the descriptor's
// bounds check), and so do the columns from row_elems on (a head narrower than the tile): their lanes carry an
// offset of 2 GiB, which no tensor reaches (the launchers check), and the sum with the offset of a tile that starts in front of the
// tensor's end cannot wrap.  The forward kernel's K tile may start up to 31 rows behind it: with rows of over 1024 elements and a tensor just under
// 2 GiB those columns wrap around to its first rows, which exist, and the scores of such keys are masked.
template <int D, int N>
struct RowCopier {
    static constexpr int UPR = D / 8, ROWS_PER_COPY = 1024 / (2 * D);
    uint32_t off[N];
    int first;
    __device__ __forceinline__ void init(int first_, long ld, int row_elems) {
        first = first_;
        const int lane = threadIdx.x & 63;
        const int lrow = lane / UPR, pos = lane % UPR;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int row = (first + i) * ROWS_PER_COPY + lrow;
            const int unit = pos ^ swz_unit<D>(row);
            off[i] = unit * 8 < row_elems ? (uint32_t)((row * ld + unit * 8) * 2) : 0x80000000u;
        }
    }
    // the tile whose first row is row0 and whose first column is col0 of the tensor rs describes (row length ld)
    __device__ __forceinline__ void issue(__amdgpu_buffer_rsrc_t rs, uint8_t *tile, long row0, long ld, long col0) const {
        const uint32_t base = (uint32_t)((row0 * ld + col0) * 2);
#pragma unroll
        for (int i = 0; i < N; ++i)
            __builtin_amdgcn_raw_ptr_buffer_load_lds(rs, (lds_void *)(tile + (first + i) * ROWS_PER_COPY * 2 * D), 16,
                                                     (int)(off[i] + base), 0, 0, 0);
    }
};
constexpr size_t MAX_TENSOR_BYTES = 0x7fff0000ull;      // what RowCopier's offsets allow

// Transposing reads.  Lane constants: 16-lane group gq = lane >> 4 forms the fragment rows (features)
// 16 (gq & 1) .. + 15 for lane half h = gq >> 1; as a source, lane j = lane & 15 of the group supplies
// the address of tile row 4 h + (j >> 2) (+ a multiple of 8), features 4 (j & 3) .. + 3 of the group's 16.
// off[2 C + SEC] holds that address for feature block C and the first or second 8 rows of 16, whose bit is in the swizzle.
template <int D>
struct TrReader {
    static constexpr int N = D / 16;
    uint32_t off[N];
    __device__ __forceinline__ void init(uint32_t lds_base) {
        const int lane = threadIdx.x & 63, gq = lane >> 4, j = lane & 15, qd = j & 3, t = j >> 2, h = gq >> 1;
        const int L = (2 * (gq & 1) + (qd >> 1)) ^ swz_unit<D>(4 * h + t);
#pragma unroll
        for (int x = 0; x < N; ++x) off[x] = lds_base + (4 * h + t) * 2 * D + (qd & 1) * 8 + ((L ^ (4 * (x >> 1)) ^ (x & 1)) << 4);
    }
    // half SEC (elements 4 SEC .. 4 SEC + 3) of the fragment of 32-row block B, MFMA M of the block, feature
    // block C of a tile at byte offset `tile` from lds_base: rows 32 B + 16 M + 8 SEC + 4 h + (0..3)
    template <int B, int M, int C, int SEC>
    __device__ __forceinline__ shortx4 read(uint32_t tile) const {
        shortx4 v;
        asm volatile("ds_read_b64_tr_b16 %0, %1 offset:%2" : "=v"(v) : "v"(off[2 * C + SEC] + tile), "n"((32 * B + 16 * M + 8 * SEC) * 2 * D));
        return v;
    }
    // the same with the tile's offset already added to the addresses (base) and a constant offset on top
    template <int B, int M, int C, int SEC, int EXTRA>
    static __device__ __forceinline__ shortx4 read_at(const uint32_t (&base)[N]) {
        constexpr int IMM = (32 * B + 16 * M + 8 * SEC) * 2 * D + EXTRA;
        static_assert(IMM < 65536, "LDS offset field");
        shortx4 v;
        asm volatile("ds_read_b64_tr_b16 %0, %1 offset:%2" : "=v"(v) : "v"(base[2 * C + SEC]), "n"(IMM));
        return v;
    }
};
__device__ __forceinline__ bf16x8 join(shortx4 lo, shortx4 hi) {
    const shortx8 v = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
    return *reinterpret_cast<const bf16x8 *>(&v);
}
// The transposing reads are written as assembly because the compiler makes the builtin wait for every
// direct-to-LDS copy in flight; their results may be used only after this wait, which names them.
#define TR_WAIT4(x) "+v"(x[0]), "+v"(x[1]), "+v"(x[2]), "+v"(x[3])
#define TR_WAIT3(x) "+v"(x[0]), "+v"(x[1]), "+v"(x[2])
#define TR_WAIT2(x) "+v"(x[0]), "+v"(x[1])
// four arrays of CB transposing reads each have landed
template <int CB, int N>
__device__ __forceinline__ void tr_wait(shortx4 (&a)[N], shortx4 (&b)[N], shortx4 (&c)[N], shortx4 (&d)[N]) {
    if constexpr (CB == 4) asm volatile("s_waitcnt lgkmcnt(0)" : TR_WAIT4(a), TR_WAIT4(b), TR_WAIT4(c), TR_WAIT4(d));
    else if constexpr (CB == 3) asm volatile("s_waitcnt lgkmcnt(0)" : TR_WAIT3(a), TR_WAIT3(b), TR_WAIT3(c), TR_WAIT3(d));
    else asm volatile("s_waitcnt lgkmcnt(0)" : TR_WAIT2(a), TR_WAIT2(b), TR_WAIT2(c), TR_WAIT2(d));
}

template <int I, int N, typename F>
__device__ __forceinline__ void static_for(F &&f) {
    if constexpr (I < N) {
        f(std::integral_constant<int, I>{});
        static_for<I + 1, N>(f);
    }
}
// LDS read of the dK/dV kernel's first wavefronts.  A read written as assembly may only be waited for in one place of the program: where two
// branches follow it, each with a wait of its own, the compiler copied the result in one of them in front of that branch's wait.
template <typename V>
__device__ __forceinline__ V lds_load(uint32_t addr) {
    return *(volatile __attribute__((address_space(3))) const V *)(uintptr_t)addr;
}
// LDS reads of its second wavefronts, written as assembly together with their waits: the compiler makes reads wait for copies in flight
// and does not count the transposing reads, so its waits come out stricter than needed.  All of them are volatile, so they are issued
// in source order, and the kernel counts that order.
template <int IMM, typename V>
__device__ __forceinline__ void lds_read16(V &dst, uint32_t addr) {
    static_assert(sizeof(V) == 16 && IMM >= 0 && IMM < 65536, "ds_read_b128");
    asm volatile("ds_read_b128 %0, %1 offset:%2" : "=v"(dst) : "v"(addr), "n"(IMM));
}
// Two wavefronts of a workgroup that share a row block (PARTS = 2): the second leaves its N values per lane in LDS, the first
// picks them up after the barrier in between.  box: XCHG_BYTES<N> bytes that belong to the pair.
template <int N>
constexpr int XCHG_BYTES = (N + 3) / 4 * 1024;
template <int CB>
__device__ __forceinline__ void put_acc(uint8_t *box, const f32x16 (&acc)[CB]) {
    f32x4 *p = reinterpret_cast<f32x4 *>(box) + (threadIdx.x & 63);
#pragma unroll
    for (int c = 0; c < CB; ++c)
#pragma unroll
        for (int i = 0; i < 4; ++i) p[(4 * c + i) * 64] = f32x4{acc[c][4 * i], acc[c][4 * i + 1], acc[c][4 * i + 2], acc[c][4 * i + 3]};
}
// acc = acc * w_own + what the other wavefront put * w_other
template <int CB>
__device__ __forceinline__ void merge_acc(const uint8_t *box, f32x16 (&acc)[CB], float w_own, float w_other) {
    const f32x4 *p = reinterpret_cast<const f32x4 *>(box) + (threadIdx.x & 63);
#pragma unroll
    for (int c = 0; c < CB; ++c)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const f32x4 v = p[(4 * c + i) * 64];
#pragma unroll
            for (int e = 0; e < 4; ++e) acc[c][4 * i + e] = acc[c][4 * i + e] * w_own + v[e] * w_other;
        }
}

// Exchange between lane l and lane l ^ 32 in one vector instruction (the two halves of a wavefront hold the two halves of
// every query's keys): after the swap the first result holds the lower half's values in both halves, the second the upper's.
__device__ __forceinline__ float max_across_halves(float v) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float sum_across_halves(float v) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}
// The forward kernel's running maximum is lazy: the reference the exponentials are taken against moves only when a
// block's maximum exceeds it by more than 2^LAZY_LOG2 (in units of the exponent), so the output accumulators are rescaled
// a few times per query instead of at almost every block; exponentials stay below 2^LAZY_LOG2, far inside fp32 and bf16 range.
// From the first block to the second it moves by any amount: the exponential of the maximum is 1 and has no rounding error, and of 64
// keys the first reference is more often the row's maximum than of 32 (l2 error of the output, 1100 causal tokens of 64 heads: 2.051e-3; lazy
// there too 2.079e-3; the maximum over 64 keys at once 2.058e-3).
constexpr float LAZY_LOG2 = 8.f;

// LDS reads of items lo .. hi - 1 of a forward block of KS items with one read each and NI - KS with two
template <int KS, int NI>
constexpr int lds_ops(int lo, int hi) {
    int n = 0;
    for (int x = lo; x < hi && x < NI; ++x) n += x < KS ? 1 : 2;
    return n;
}

}  // namespace

}  // namespace mmt
