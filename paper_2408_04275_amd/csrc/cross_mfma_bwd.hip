// Backward of attention from runs of queries to ranges of keys on the matrix cores (bf16 in, fp32 accumulate): the layout of
// cross_mfma.hip, two kernels.  dQ holds one row per lane and walks the keys of its run; it also writes -D, D = rowsum(dO * O).
// dK/dV holds one key per lane and walks the rows that see its keys.  For that the keys are cut wherever a run's range begins or ends
// (make_plan): all keys of a tile are seen by the same runs, which follow one another, so again nothing is masked.  Keys that several runs
// see, and heads of a group, are summed in registers, in the order of the runs: nothing needs atomics.  P and dS are rounded to bf16 as operands of their products with dO, Q
// and K, for the reason that cross_mfma.hip gives; each gradient is off by 0.0022 to 0.0024 of its norm.
#include "cross_tiles.h"
#include <algorithm>

namespace mmt {

namespace {

// A wavefront's share of 64 rows on their way into LDS: copies first .. first + N - 1 of 1 KiB each
template <int D, int N>
__device__ __forceinline__ void copy_rows_part(const bf16_t *p, long ld, int dh, const Rows &at, const Group &g, uint8_t *tile, int first) {
    constexpr int UPR = D / 8, PER = 1024 / (2 * D);
    const __amdgpu_buffer_rsrc_t rs = __builtin_amdgcn_make_buffer_rsrc(const_cast<bf16_t *>(p + at.t * ld), 0, 0x7fff0000, 0x00020000);
    const int lane = threadIdx.x & 63, lrow = lane / UPR, pos = lane % UPR;
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const int row = (first + i) * PER + lrow, unit = pos ^ swz_unit<D>(row);
        const uint32_t there = (at.offset(g, row, ld, dh) + unit * 8) * 2u, off = row < at.left && unit * 8 < dh ? there : 0x80000000u;
        __builtin_amdgcn_raw_ptr_buffer_load_lds(rs, (lds_void *)(tile + (first + i) * PER * 2 * D), 16, (int)off, 0, 0, 0);
    }
}

template <int D> constexpr int STAGE32 = 32 * (4 * D + 16);
// a wavefront's 32 keys' results, unscaled, as fp32 rows of a workgroup's part
template <int D, int CB>
__device__ __forceinline__ void store_part(uint8_t *stage, const f32x16 (&acc)[CB], float *dst, long ld, int rows, int dh) {
    constexpr int RS = 4 * D + 16, LPR = D / 4, RPI = 64 / LPR;
    const int lane = threadIdx.x & 63, half = lane >> 5, l32 = lane & 31;
#pragma unroll
    for (int c = 0; c < CB; ++c)
#pragma unroll
        for (int gq = 0; gq < 4; ++gq)
            *reinterpret_cast<f32x4 *>(stage + l32 * RS + (32 * c + 8 * gq + 4 * half) * 4) =
                f32x4{acc[c][4 * gq], acc[c][4 * gq + 1], acc[c][4 * gq + 2], acc[c][4 * gq + 3]};
    const int r0 = lane / LPR, cb = (lane % LPR) * 4;
    const __amdgpu_buffer_rsrc_t rs = __builtin_amdgcn_make_buffer_rsrc(dst, 0, 0x7fff0000, 0x00020000);
#pragma unroll
    for (int i0 = 0; i0 < 32 / RPI; i0 += 8) {
        u32x4 v[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = *reinterpret_cast<const u32x4 *>(stage + ((i0 + i) * RPI + r0) * RS + cb * 4);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int r = (i0 + i) * RPI + r0;
            const uint32_t off = (uint32_t)(r * (int)ld + cb) * 4u;
            __builtin_amdgcn_raw_buffer_store_b128(v[i], rs, (int)(r < rows && cb < dh ? off : 0x80000000u), 0, 0);
        }
    }
}

// ---- dQ --------------------------------------------------------------------------------------------------------------------
// Four wavefronts of 32 rows, two workgroups a compute unit; one wavefront for many short runs, where it is faster (see cross_bwd_plan).  Eight were nowhere faster than four and
// are not built: us, 128 / 256 rows, both backward kernels: 4096 tokens of 32 heads of 128, on 8 in one run of 8192 keys 1785 / 1792, four runs of 2304 603 / 635; 2111 tokens in 61 runs of 300 237 / 284.
// 8192 tokens of 32 heads of 128 in 12 runs of 1152 keys 250 us (0.64 PFLOP/s): Q, dO, O and dQ alone take 47 (5.7 TB/s), a step of 64 keys of both workgroups 2.6 (1.24 PFLOP/s),
// bound by the matrix cores.  Q and dO on their way together instead of one after the other, and tiles of 32 keys: no difference.
// LDS: two slots of a K and a V tile; the Q, dO and O rows stand in the second slot, one after the other.
template <int WAVES> constexpr int DQ_STEP = WAVES == 4 ? 64 : 32;
template <int D, int WAVES> constexpr int DQ_LDS = 2 * 2 * DQ_STEP<WAVES> * D * 2;

template <int D, int KS, int CB, int WAVES>
__global__ __launch_bounds__(64 * WAVES, 2) void cross_dq_kernel(CrossArgs a) {
    constexpr int ROWS = 32 * WAVES, STEP = DQ_STEP<WAVES>, TILE = STEP * D * 2, SLOT = 2 * TILE, COPIES = TILE / 1024 / WAVES;
    extern __shared__ __attribute__((aligned(16))) uint8_t smem[];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), half = lane >> 5, l32 = lane & 31;
    int block = blockIdx.x;
    if (a.n_tiles > 0 && block-- == 0) { make_plan<64 * WAVES>(a, (int *)smem); return; }
    const int head = block % a.nkv, dh = a.d;
    const Item it = find_item(a, block / a.nkv, ROWS, a.chunk);
    const int parts = a.chunk ? max((it.hi - it.lo + a.chunk - 1) / a.chunk, 1) : 1, part = it.index % parts;
    const Group g(a);
    const Rows mine(it, g, it.index / parts * ROWS + wave * 32);
    const int kbeg = it.lo + part * a.chunk, kend = !a.dq ? kbeg : parts > 1 ? min(kbeg + a.chunk, it.hi) : it.hi;
    const bf16_t *const K = (const bf16_t *)a.k + (long)head * dh, *const V = (const bf16_t *)a.v + (long)head * dh;
    const long col = (long)head * g.n * dh;

    RowCopier<D, COPIES> cpk, cpv;
    cpk.init(wave * COPIES, a.ldk, dh);
    cpv.init(wave * COPIES, a.ldv, dh);
    auto copy_kv = [&](uint8_t *slot, int kt) {
        cpk.issue(rows_rsrc(K, kt, a.ldk, kend - kt, dh), slot, 0, 0, 0);
        cpv.issue(rows_rsrc(V, kt, a.ldv, kend - kt, dh), slot + TILE, 0, 0, 0);
    };
    bf16x8 qf[KS], dof[KS];
    float Dq = 0.f;
    {
        uint8_t *const stage = smem + SLOT + wave * ROWS32<D>;
        copy_rows<D>((const bf16_t *)a.q + col, a.ldq, dh, mine, g, stage);
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) qf[ks] = frag_k<D>(stage, l32, ks, half);
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");           // read: dO may take the place
        copy_rows<D>((const bf16_t *)a.d_o + col, a.lddo, dh, mine, g, stage);
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) dof[ks] = frag_k<D>(stage, l32, ks, half);
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        copy_rows<D>((const bf16_t *)a.o + col, a.ldo, dh, mine, g, stage);
        if (kbeg < kend) copy_kv(smem, kbeg);
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
            const bf16x8 of = frag_k<D>(stage, l32, ks, half);
            const uint4 w = *reinterpret_cast<const uint4 *>(&dof[ks]), x = *reinterpret_cast<const uint4 *>(&of);
            const uint32_t dw[4] = {w.x, w.y, w.z, w.w}, ow[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                Dq += __uint_as_float(dw[e] << 16) * __uint_as_float(ow[e] << 16);
                Dq += __uint_as_float(dw[e] & 0xffff0000u) * __uint_as_float(ow[e] & 0xffff0000u);
            }
        }
    }
    Dq += __shfl_xor(Dq, 32, 64);
    float lse2 = 0.f;                                  // log-sum-exp in log2 units
    if (l32 < mine.left) {
        const int tok = g.token(mine.j + l32), h = head * g.n + mine.j + l32 - tok * g.n;
        const long at = (long)h * a.Tq + mine.t + tok;
        lse2 = a.lse[at] * LOG2E;
        if (half == 0 && part == 0) a.D[at] = -Dq;
    }
    if (!a.dq) return;
    // with 64-wide heads dP - D comes out of the matrix core (see attn_mfma.hip)
    constexpr bool D_IN_MFMA = D <= 64;
    f32x16 negD;
#pragma unroll
    for (int i = 0; i < 16; ++i) negD[i] = D_IN_MFMA ? -Dq : 0.f;
    f32x16 dq[CB];
#pragma unroll
    for (int c = 0; c < CB; ++c) dq[c] = zero16();
    const float sl2 = a.scale * LOG2E;
    TrReader<D> tr;
    tr.init((uint32_t)(uintptr_t)(lds_void *)smem);

    int slot = 0;
    for (int kt = kbeg; kt < kend; kt += STEP, slot ^= 1) {
        const uint8_t *sK = smem + slot * SLOT, *sV = sK + TILE;
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");             // this step's tiles have landed
        lds_barrier();                                               // ... and everyone is done with the other slot
        if (kt + STEP < kend) copy_kv(smem + (slot ^ 1) * SLOT, kt + STEP);
        auto block = [&](auto B_) {
            constexpr int b = decltype(B_)::value;
            const int kb = kt + 32 * b;
            if (kb >= kend || mine.left <= 0) return;
            f32x16 s = zero16(), dp = negD;
#pragma unroll
            for (int ks = 0; ks < KS; ++ks) {
                s = MFMA(frag_k<D>(sK, 32 * b + l32, ks, half), qf[ks], s);
                dp = MFMA(frag_k<D>(sV, 32 * b + l32, ks, half), dof[ks], dp);
            }
            // K^T fragments of this block: [MFMA m][feature block c], two halves each
            shortx4 t0[4], t1[4], t2[4], t3[4];                      // (m, sec) = (0,0), (0,1), (1,0), (1,1)
            const uint32_t tile = slot * SLOT;
            static_for<0, CB>([&](auto C_) {
                constexpr int c = decltype(C_)::value;
                t0[c] = tr.template read<b, 0, c, 0>(tile); t1[c] = tr.template read<b, 0, c, 1>(tile);
                t2[c] = tr.template read<b, 1, c, 0>(tile); t3[c] = tr.template read<b, 1, c, 1>(tile);
            });
            float ds[16];
            auto softmax = [&](auto MASK_) {
                const int left = kend - kb - 4 * half;
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    float p = __builtin_amdgcn_exp2f(fmaf(s[i], sl2, -lse2));
                    if (decltype(MASK_)::value) p = 8 * (i >> 2) + (i & 3) < left ? p : 0.f;
                    ds[i] = D_IN_MFMA ? p * dp[i] : p * (dp[i] - Dq);
                }
            };
            if (kb + 32 <= kend) softmax(std::false_type{});
            else softmax(std::true_type{});
            tr_wait<CB>(t0, t1, t2, t3);
            const bf16x8 ds0 = pack8(ds), ds1 = pack8(ds + 8);
#pragma unroll
            for (int c = 0; c < CB; ++c) {
                dq[c] = MFMA(join(t0[c], t1[c]), ds0, dq[c]);
                dq[c] = MFMA(join(t2[c], t3[c]), ds1, dq[c]);
            }
        };
        block(std::integral_constant<int, 0>{});
        if constexpr (STEP > 32) block(std::integral_constant<int, 1>{});
    }
    lds_barrier();                                     // the tiles are done with: LDS now stages the output rows
    if (parts > 1) store_part<D, CB>(smem + wave * STAGE32<D>, dq, a.part + ((size_t)block * ROWS + wave * 32) * dh, dh, mine.left, dh);
    else store_rows_at<D, CB>(smem + wave * STAGE<D>, dq, a.scale, (bf16_t *)a.dq + col, a.lddq, dh, mine, g);
}

// 64 values of a [heads, Tq] array, those of a step's rows, into LDS
__device__ __forceinline__ void copy_stats(const float *x, const CrossArgs &a, int head, const Rows &at, const Group &g, uint8_t *to) {
    const int lane = threadIdx.x & 63, tok = g.token(at.j + lane), h = at.j + lane - tok * g.n;
    const __amdgpu_buffer_rsrc_t rs =
        __builtin_amdgcn_make_buffer_rsrc(const_cast<float *>(x + (long)head * g.n * a.Tq + at.t), 0, 0x7fff0000, 0x00020000);
    const uint32_t off = lane < at.left ? (uint32_t)(h * a.Tq + tok) * 4u : 0x80000000u;
    __builtin_amdgcn_raw_ptr_buffer_load_lds(rs, (lds_void *)to, 4, (int)off, 0, 0, 0);
}

template <int D, int CB>
__device__ __forceinline__ void store_dkv(const CrossArgs &a, uint8_t *smem, int wave, int head, int key, int rows, const f32x16 (&dk)[CB], const f32x16 (&dv)[CB]) {
    const int dh = a.d, nk = a.nkv * dh;
    if (a.parts > 1) {
        float *out = a.dkv_part + ((size_t)blockIdx.y * a.Tk + key) * 2 * nk + head * dh;
        store_part<D, CB>(smem + wave * STAGE32<D>, dk, out, 2 * nk, rows, dh);
        store_part<D, CB>(smem + wave * STAGE32<D>, dv, out + nk, 2 * nk, rows, dh);
        return;
    }
    const Group one(1);
    Rows at;
    at.t = key; at.j = 0; at.left = rows;
    store_rows_at<D, CB>(smem + wave * STAGE<D>, dv, 1.f, (bf16_t *)a.dv + head * dh, a.lddv, dh, at, one);
    store_rows_at<D, CB>(smem + wave * STAGE<D>, dk, a.scale, (bf16_t *)a.dk + head * dh, a.lddk, dh, at, one);
}

// ---- dK, dV for heads wider than 64 features ----------------------------------------------------------------------------------
// As in attn_mfma.hip: 32 keys belong to a pair of wavefronts on one SIMD, of which the first turns 32 rows at a time into P and dS
// and the second adds dO^T P and Q^T dS, one block behind; P and dS go through LDS, rows round three slots of 64.  The same pack as above 355 us (0.60 PFLOP/s):
// 1.9 us a step (1.13 PFLOP/s), bound by the matrix cores, and 5 us at the beginning and end of each of a compute unit's 14 tiles, with nothing beside it (LDS holds one
// workgroup).
template <int D> constexpr int DKV_SLOT = 2 * STEP_ROWS * D * 2 + 2 * STEP_ROWS * 4;        // Q tile, dO tile, lse[64], D[64]
constexpr int PDS_BYTES = 4 * 1024;                                                        // P and dS of one block of one pair
template <int D> constexpr int DKV_PAIR_LDS = 3 * DKV_SLOT<D> + 2 * 4 * PDS_BYTES;

template <int D, int KS, int CB>
__global__ __launch_bounds__(512, 2) void cross_dkv_kernel(CrossArgs a) {
    constexpr int TILE = STEP_ROWS * D * 2, SLOT = DKV_SLOT<D>, COPIES = TILE / 1024 / 4;   // copies per second wavefront and tile
    extern __shared__ __attribute__((aligned(16))) uint8_t smem[];
    const int lane = threadIdx.x & 63, wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), half = lane >> 5, l32 = lane & 31;
    const int pair = wv & 3, head = blockIdx.x % a.nkv, dh = a.d;
    const KeyTile kt = find_tile(a, blockIdx.x / a.nkv);
    const int key = kt.key + pair * 32, n_steps = kt.steps;
    const bool live = key < kt.end;                     // (a pair behind the last key copies its share of the rows and no more)
    const uint32_t lds0 = (uint32_t)(uintptr_t)(lds_void *)smem;
    const uint32_t box0 = lds0 + 3 * SLOT + pair * PDS_BYTES + lane * 16;        // this lane's part of the pair's first buffer
    auto next_slot = [](uint32_t tile) { return tile == 2 * SLOT ? 0u : tile + SLOT; };
    const int4 *const steps = a.steps + kt.step;

    if (wv < 4) {
        if (n_steps == 0) { lds_barrier(); return; }
        bf16x8 kf[KS], vf[KS];                         // K and V rows as the MFMA's column operands
        {
            static_assert(4 * ROWS32<D> <= SLOT && 4 * ROWS32<D> <= 8 * PDS_BYTES, "room for the staged K and V rows");
            RowCopier<D, ROWS32<D> / 1024> cpk, cpv;
            cpk.init(0, a.ldk, dh);
            cpv.init(0, a.ldv, dh);
            uint8_t *stage_k = smem + 3 * SLOT + pair * ROWS32<D>, *stage_v = smem + 2 * SLOT + pair * ROWS32<D>;
            cpk.issue(rows_rsrc((const bf16_t *)a.k + head * dh, key, a.ldk, min(kt.end - key, 32), dh), stage_k, 0, 0, 0);
            cpv.issue(rows_rsrc((const bf16_t *)a.v + head * dh, key, a.ldv, min(kt.end - key, 32), dh), stage_v, 0, 0, 0);
            asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
#pragma unroll
            for (int ks = 0; ks < KS; ++ks) {
                kf[ks] = frag_k<D>(stage_k, l32, ks, half);
                vf[ks] = frag_k<D>(stage_v, l32, ks, half);
            }
        }
        const float sl2 = a.scale * LOG2E;
        uint32_t f0[KS];
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) f0[ks] = lds0 + (l32 * (D / 8) + ((2 * ks + half) ^ swz_unit<D>(l32))) * 16;
        const uint32_t l0 = lds0 + 2 * TILE + half * 16;
        uint32_t tile = 0;                              // LDS offset of the step's slot
        auto block = [&](auto B_) {
            constexpr int b = decltype(B_)::value;
            constexpr int NF = 2 * KS, AHEAD = 8;
            bf16x8 fr[NF];
            f32x4 l4[4], d4[4];
            uint32_t fa, la = l0 + tile;
            asm volatile("" : "+v"(la));
            auto issue = [&](auto I_) {
                constexpr int i = decltype(I_)::value;
                if constexpr (i < NF) {
                    if constexpr ((i & 1) == 0) { fa = f0[i >> 1] + tile; asm volatile("" : "+v"(fa)); }      // (one address for both reads)
                    fr[i] = lds_load<bf16x8>(fa + ((i & 1) * TILE + b * 64 * D));
                } else if constexpr (((i - NF) & 1) == 0) l4[(i - NF) / 2] = lds_load<f32x4>(la + (b * 128 + (i - NF) / 2 * 32));
                else d4[(i - NF) / 2] = lds_load<f32x4>(la + (b * 128 + (i - NF) / 2 * 32 + STEP_ROWS * 4));
            };
            static_for<0, AHEAD>([&](auto I_) { issue(I_); });
            __builtin_amdgcn_sched_barrier(0);
            f32x16 s = zero16(), dp = zero16();
            static_for<0, NF>([&](auto J_) {
                constexpr int j = decltype(J_)::value;
                if constexpr ((j & 1) == 0) s = MFMA(fr[j], kf[j >> 1], s);
                else dp = MFMA(fr[j], vf[j >> 1], dp);
                issue(std::integral_constant<int, j + AHEAD>{});
                __builtin_amdgcn_sched_barrier(0);
            });
            uint32_t pp[8], dd[8];
            static_for<0, 4>([&](auto Q_) {
                constexpr int gq = decltype(Q_)::value;
                float p[4], ds[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    p[e] = __builtin_amdgcn_exp2f(fmaf(s[4 * gq + e], sl2, -l4[gq][e] * LOG2E));
                    ds[e] = p[e] * (dp[4 * gq + e] + d4[gq][e]);                 // the D array holds -D
                }
                pp[2 * gq] = pack_bf16x2(p[0], p[1]); pp[2 * gq + 1] = pack_bf16x2(p[2], p[3]);
                dd[2 * gq] = pack_bf16x2(ds[0], ds[1]); dd[2 * gq + 1] = pack_bf16x2(ds[2], ds[3]);
            });
            auto *box = reinterpret_cast<__attribute__((address_space(3))) rawx4 *>((uintptr_t)(box0 + b * 4 * PDS_BYTES));
            box[0] = rawx4{pp[0], pp[1], pp[2], pp[3]};
            box[64] = rawx4{pp[4], pp[5], pp[6], pp[7]};
            box[128] = rawx4{dd[0], dd[1], dd[2], dd[3]};
            box[192] = rawx4{dd[4], dd[5], dd[6], dd[7]};
        };
        int left = entry_of(steps, 0).z;
        for (int step = 0; step < n_steps; ++step) {
            const int now = left;
            if (step + 1 < n_steps) left = entry_of(steps, step + 1).z;
            lds_barrier();
            if (live) block(std::integral_constant<int, 0>{});
            lds_barrier();
            if (now > 32 && live) block(std::integral_constant<int, 1>{});
            tile = next_slot(tile);
        }
        lds_barrier();                                 // the last block's P and dS are there
        lds_barrier();                                 // the tiles are done with
        return;
    }

    // ---- the second wavefront of a pair
    f32x16 dk[CB], dv[CB];
#pragma unroll
    for (int c = 0; c < CB; ++c) { dk[c] = zero16(); dv[c] = zero16(); }
    if (n_steps > 0) {
        const Group g(a);
        const bf16_t *const Q = (const bf16_t *)a.q + (long)head * g.n * dh, *const dO = (const bf16_t *)a.d_o + (long)head * g.n * dh;
        // each copies a quarter of the Q tile and of the dO tile; the first two also fetch the log-sum-exps and the D values
        auto copy_q = [&](uint32_t slot, const Rows &at) { copy_rows_part<D, COPIES>(Q, a.ldq, dh, at, g, smem + slot, pair * COPIES); };
        auto copy_do = [&](uint32_t slot, const Rows &at) {
            copy_rows_part<D, COPIES>(dO, a.lddo, dh, at, g, smem + slot + TILE, pair * COPIES);
            if (pair < 2) copy_stats(pair == 0 ? a.lse : a.D, a, head, at, g, smem + slot + 2 * TILE + pair * STEP_ROWS * 4);
        };
        TrReader<D> tr;
        tr.init(lds0);
        auto block = [&](auto B_, uint32_t tile) {
            constexpr int b = decltype(B_)::value;
            constexpr int NG = 2 * CB;
            bf16x8 pf[2], dsf[2];
            shortx4 o[NG][2], q[NG][2];
            const uint32_t box = box0 + b * 4 * PDS_BYTES;
            uint32_t trc[TrReader<D>::N];
#pragma unroll
            for (int x = 0; x < TrReader<D>::N; ++x) trc[x] = tr.off[x] + tile;
            lds_read16<0>(pf[0], box); lds_read16<2048>(dsf[0], box);
            lds_read16<1024>(pf[1], box); lds_read16<3 * 1024>(dsf[1], box);
            auto issue = [&](auto G_) {
                constexpr int gi = decltype(G_)::value, m = gi / CB, c = gi % CB;
                o[gi][0] = TrReader<D>::template read_at<b, m, c, 0, TILE>(trc); o[gi][1] = TrReader<D>::template read_at<b, m, c, 1, TILE>(trc);
                q[gi][0] = TrReader<D>::template read_at<b, m, c, 0, 0>(trc); q[gi][1] = TrReader<D>::template read_at<b, m, c, 1, 0>(trc);
            };
            static_for<0, 3>([&](auto G_) { issue(G_); });
            static_for<0, NG>([&](auto G_) {
                constexpr int gi = decltype(G_)::value, m = gi / CB, c = gi % CB, LEFT = NG - 1 - gi < 2 ? NG - 1 - gi : 2;
                asm volatile("s_waitcnt lgkmcnt(%4)" : TR_WAIT2(o[gi]), TR_WAIT2(q[gi]) : "n"(4 * LEFT));
                if constexpr (gi == 0) asm volatile("" : "+v"(pf[0]), "+v"(dsf[0]), "+v"(pf[1]), "+v"(dsf[1]));
                dv[c] = MFMA(join(o[gi][0], o[gi][1]), pf[m], dv[c]);
                dk[c] = MFMA(join(q[gi][0], q[gi][1]), dsf[m], dk[c]);
                if constexpr (gi + 3 < NG) issue(std::integral_constant<int, gi + 3>{});
            });
        };
        // rows of steps t, t + 1 (copied) and t + 2 (next to be copied, its entry requested a step ahead)
        int4 entry = entry_of(steps, 0), second = n_steps > 1 ? entry_of(steps, 1) : entry;
        Rows now = rows_of(entry), next = rows_of(second), after = now;
        if (n_steps > 2) entry = entry_of(steps, 2);
        copy_q(0, now);
        copy_do(0, now);
        if (n_steps > 1) {
            copy_q(SLOT, next);
            copy_do(SLOT, next);
        }
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        // Barrier 2 t stands in front of the first wavefront's block 0 of step t (tile t has landed, block 1 of step t - 1 is in its
        // buffer), barrier 2 t + 1 in front of its block 1.  Behind the latter nobody reads tile t - 1 any more: its slot is tile t + 2's,
        // whose Q rows are requested there and whose dO rows behind the next barrier.
        uint32_t tile = 0, before = 2 * SLOT;          // slots of tiles t and t - 1 (which is tile t + 2's)
        int left_before = 0;
        for (int step = 0; step < n_steps; ++step) {
            lds_barrier();
            if (step > 0) {
                if (step + 1 < n_steps) copy_do(next_slot(tile), next);
                if (left_before > 32 && live) block(std::integral_constant<int, 1>{}, before);
            }
            lds_barrier();
            if (step + 2 < n_steps) {
                after = rows_of(entry);
                if (step + 3 < n_steps) entry = entry_of(steps, step + 3);
                copy_q(before, after);
            }
            if (live) block(std::integral_constant<int, 0>{}, tile);
            // tile t + 1 has landed; the copies of Q for tile t + 2 may be in flight (memory operations retire in order)
            if (step + 2 < n_steps) asm volatile("s_waitcnt vmcnt(%0)" ::"n"(COPIES) : "memory");
            else asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
            before = tile;
            tile = next_slot(tile);
            left_before = now.left;
            now = next;
            next = after;
        }
        lds_barrier();
        if (left_before > 32 && live) block(std::integral_constant<int, 1>{}, before);
    }
    lds_barrier();                                     // the tiles are done with: LDS now stages the output rows
    store_dkv<D, CB>(a, smem, pair, head, key, kt.end - key, dk, dv);
}

// ---- dK, dV for heads of up to 64 features --------------------------------------------------------------------------------------
// A block's scores, its exponentials and its products one after the other; four wavefronts of 32 keys, two LDS slots, two workgroups per compute unit.
template <int D> constexpr int DKV_PLAIN_LDS = 2 * DKV_SLOT<D> + 4 * 2 * ROWS32<D>;

template <int D>
__global__ __launch_bounds__(256, 2) void cross_dkv_plain_kernel(CrossArgs a) {
    constexpr int KS = D / 16, CB = D / 32;
    constexpr int TILE = STEP_ROWS * D * 2, SLOT = DKV_SLOT<D>, COPIES = TILE / 1024 / 4;
    extern __shared__ __attribute__((aligned(16))) uint8_t smem[];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), half = lane >> 5, l32 = lane & 31;
    const int head = blockIdx.x % a.nkv, dh = a.d;
    const KeyTile kt = find_tile(a, blockIdx.x / a.nkv);
    const int key = kt.key + wave * 32, n_steps = kt.steps;
    f32x16 dk[CB], dv[CB];
#pragma unroll
    for (int c = 0; c < CB; ++c) { dk[c] = zero16(); dv[c] = zero16(); }
    if (n_steps > 0) {
        const Group g(a);
        const bf16_t *const Q = (const bf16_t *)a.q + (long)head * g.n * dh, *const dO = (const bf16_t *)a.d_o + (long)head * g.n * dh;
        const int4 *const steps = a.steps + kt.step;
        const float sl2 = a.scale * LOG2E;
        auto copy_tile = [&](uint8_t *slot, const Rows &at) {
            copy_rows_part<D, COPIES>(Q, a.ldq, dh, at, g, slot, wave * COPIES);
            copy_rows_part<D, COPIES>(dO, a.lddo, dh, at, g, slot + TILE, wave * COPIES);
            if (wave < 2) copy_stats(wave == 0 ? a.lse : a.D, a, head, at, g, slot + 2 * TILE + wave * STEP_ROWS * 4);
        };
        TrReader<D> tr;
        tr.init((uint32_t)(uintptr_t)(lds_void *)smem);
        bf16x8 kf[KS], vf[KS];
        Rows now = rows_of(entry_of(steps, 0));
        {
            RowCopier<D, ROWS32<D> / 1024> cpk, cpv;
            cpk.init(0, a.ldk, dh);
            cpv.init(0, a.ldv, dh);
            uint8_t *stage_k = smem + 2 * SLOT + wave * 2 * ROWS32<D>, *stage_v = stage_k + ROWS32<D>;
            cpk.issue(rows_rsrc((const bf16_t *)a.k + head * dh, key, a.ldk, min(kt.end - key, 32), dh), stage_k, 0, 0, 0);
            cpv.issue(rows_rsrc((const bf16_t *)a.v + head * dh, key, a.ldv, min(kt.end - key, 32), dh), stage_v, 0, 0, 0);
            copy_tile(smem, now);
            asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
#pragma unroll
            for (int ks = 0; ks < KS; ++ks) {
                kf[ks] = frag_k<D>(stage_k, l32, ks, half);
                vf[ks] = frag_k<D>(stage_v, l32, ks, half);
            }
        }
        int4 entry = n_steps > 1 ? entry_of(steps, 1) : make_int4(0, 0, 0, 0);
        int slot = 0;
        for (int step = 0; step < n_steps; ++step, slot ^= 1) {
            const uint8_t *sQ = smem + slot * SLOT, *sdO = sQ + TILE;
            const float *sLse = reinterpret_cast<const float *>(sQ + 2 * TILE), *sD = sLse + STEP_ROWS;
            const int left = now.left;
            asm volatile("s_waitcnt vmcnt(0)" ::: "memory");             // this step's tiles have landed
            lds_barrier();                                               // ... and everyone is done with the other slot
            if (step + 1 < n_steps) {
                now = rows_of(entry);
                if (step + 2 < n_steps) entry = entry_of(steps, step + 2);
                copy_tile(smem + (slot ^ 1) * SLOT, now);
            }
            auto block = [&](auto B_) {
                constexpr int b = decltype(B_)::value;
                if (32 * b >= left || key >= kt.end) return;
                f32x16 s = zero16(), dp = zero16();
#pragma unroll
                for (int ks = 0; ks < KS; ++ks) {
                    s = MFMA(frag_k<D>(sQ, 32 * b + l32, ks, half), kf[ks], s);
                    dp = MFMA(frag_k<D>(sdO, 32 * b + l32, ks, half), vf[ks], dp);
                }
                const uint32_t tq = slot * SLOT, tdo = tq + TILE;
                shortx4 o[2][CB][2], q[2][CB][2];
                static_for<0, 2 * CB>([&](auto X_) {
                    constexpr int x = decltype(X_)::value, m = x / CB, c = x % CB;
                    o[m][c][0] = tr.template read<b, m, c, 0>(tdo); o[m][c][1] = tr.template read<b, m, c, 1>(tdo);
                    q[m][c][0] = tr.template read<b, m, c, 0>(tq); q[m][c][1] = tr.template read<b, m, c, 1>(tq);
                });
                float p[16], ds[16];
#pragma unroll
                for (int gq = 0; gq < 4; ++gq) {
                    const int r0 = 32 * b + 8 * gq + 4 * half;        // 4 consecutive rows
                    const float4 l4 = *reinterpret_cast<const float4 *>(sLse + r0);
                    const float4 d4 = *reinterpret_cast<const float4 *>(sD + r0);
                    const float lv[4] = {l4.x, l4.y, l4.z, l4.w}, dvv[4] = {d4.x, d4.y, d4.z, d4.w};
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const int i = 4 * gq + e;
                        p[i] = __builtin_amdgcn_exp2f(fmaf(s[i], sl2, -lv[e] * LOG2E));
                        ds[i] = p[i] * (dp[i] + dvv[e]);               // the D array holds -D
                    }
                }
                const bf16x8 pf[2] = {pack8(p), pack8(p + 8)}, dsf[2] = {pack8(ds), pack8(ds + 8)};
                static_for<0, 2 * CB>([&](auto X_) {
                    constexpr int x = decltype(X_)::value, m = x / CB, c = x % CB;
                    lds_wait<0>(o[m][c][0]); lds_wait<0>(o[m][c][1]);
                    lds_wait<0>(q[m][c][0]); lds_wait<0>(q[m][c][1]);
                });
                static_for<0, 2 * CB>([&](auto X_) {
                    constexpr int x = decltype(X_)::value, m = x / CB, c = x % CB;
                    dv[c] = MFMA(join(o[m][c][0], o[m][c][1]), pf[m], dv[c]);
                    dk[c] = MFMA(join(q[m][c][0], q[m][c][1]), dsf[m], dk[c]);
                });
            };
            block(std::integral_constant<int, 0>{});
            block(std::integral_constant<int, 1>{});
        }
    }
    lds_barrier();                                     // the tiles are done with: LDS now stages the output rows
    store_dkv<D, CB>(a, smem, wave, head, key, kt.end - key, dk, dv);
}

template <int D, int KS, int CB, int WAVES>
hipError_t launch_dq(const CrossArgs &a, int items, hipStream_t st) {
    static std::atomic<bool> done{false};
    constexpr int LDS = std::max({DQ_LDS<D, WAVES>, WAVES * STAGE32<D>, PLAN_LDS});
    const hipError_t e = set_smem(done, cross_dq_kernel<D, KS, CB, WAVES>, LDS);
    if (e != hipSuccess) return e;
    cross_dq_kernel<D, KS, CB, WAVES><<<items * a.nkv + (a.n_tiles > 0), 64 * WAVES, LDS, st>>>(a);
    if constexpr (WAVES == 4)                            // (with fewer there are workgroups enough)
        if (a.chunk) cross_dq_sum_kernel<bf16_t, 128><<<items * a.nkv, 256, 0, st>>>(a);
    return hipGetLastError();
}

template <int D, int KS, int CB>
hipError_t launch_bwd(const CrossArgs &a, const CrossBwdPlan &p, hipStream_t st) {
    hipError_t e = hipSuccess;
    if (p.items || a.n_tiles) e = p.rows == FEW_ROWS ? launch_dq<D, KS, CB, 1>(a, p.items, st) : launch_dq<D, KS, CB, 4>(a, p.items, st);
    if (e != hipSuccess || !a.n_tiles) return e;
    static std::atomic<bool> done{false};
    const dim3 grid(p.tiles * a.nkv, a.parts);
    if constexpr (D <= 64) {
        constexpr int LDS = std::max(DKV_PLAIN_LDS<D>, 4 * STAGE32<D>);
        if ((e = set_smem(done, cross_dkv_plain_kernel<D>, LDS)) != hipSuccess) return e;
        cross_dkv_plain_kernel<D><<<grid, 256, LDS, st>>>(a);
    } else {
        static_assert(4 * STAGE32<D> <= DKV_PAIR_LDS<D>, "room for the staged fp32 rows");
        if ((e = set_smem(done, cross_dkv_kernel<D, KS, CB>, DKV_PAIR_LDS<D>)) != hipSuccess) return e;
        cross_dkv_kernel<D, KS, CB><<<grid, 512, DKV_PAIR_LDS<D>, st>>>(a);
    }
    if (a.parts > 1) cross_dkv_sum_kernel<bf16_t><<<ceil_div((long)a.Tk * (2 * a.nkv * a.d / 4), 256), 256, 0, st>>>(a);
    return hipGetLastError();
}

}  // namespace

hipError_t cross_mfma_bwd(const CrossArgs &a, const CrossBwdPlan &p, hipStream_t st) {
    return a.d <= 64 ? launch_bwd<64, 4, 2>(a, p, st) : a.d <= 80 ? launch_bwd<128, 5, 3>(a, p, st) : a.d <= 96 ? launch_bwd<128, 6, 3>(a, p, st)
                                                                                                          : launch_bwd<128, 8, 4>(a, p, st);
}

}  // namespace mmt
