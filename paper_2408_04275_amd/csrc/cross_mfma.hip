// Attention of runs of queries to ranges of keys on the gfx950 matrix cores (bf16 in, fp32 accumulate).
//
// All tokens of a run see the same keys, and the query heads of a group share them.  So the rows of a tile are (token, head of the group)
// pairs of ONE run (or of neighbouring runs that see the same keys) and key/value head -- row r is token r / group, head r % group -- and what a workgroup
// walks is the run's keys and nothing else: no row has a mask of its own, only the last block of keys ends early.  Rows and keys that do not exist are read as
// zeros (the bounds of the buffer descriptor), so nothing that belongs to others, an infinity or NaN in the next run's keys, can enter a product.
//
// Scores are computed transposed, as in attn_mfma.hip: a lane holds 16 keys of ONE row per block of 32 keys.
//
// The probabilities are rounded to bf16, as operands of their product with V: in fp32 that product would run at a tenth of the rate (153 against 1540 TFLOP/s), and as
// two bf16 operands, value and remainder, be done twice.  The row's sum takes them unrounded.  O is off by 0.0022 to 0.0024 of its norm; rounded once at the end, by 0.0017.
#include "cross_tiles.h"
#include <algorithm>

namespace mmt {

namespace {

// ---- forward, many rows ------------------------------------------------------------------------------------------------
// WAVES wavefronts x 32 rows, keys 64 at a time through two LDS slots.  Each wavefront works one block of 32 keys ahead, as
// attn_mfma.hip's forward kernel does: the next block's scores are multiplied between the exponentials of the current one, and a
// step's K tile stands one block further on than its V tile.  8192 tokens of 32 heads of 128 in 12 runs of 1152 keys 183 us (0.81 PFLOP/s, 26 us of it without any key:
// Q in, O out), 4096 of 32 heads on 8 in one run of 8192 keys 475 us (1.16): bound by the matrix cores and the exponentials beside them.
template <int D, int WAVES> constexpr int FWD_LDS = 2 * 2 * KEYS * D * 2 + (WAVES == 8 ? 9 : 1) * ROWS32<D>;

template <int D, int KS, int CB, int WAVES>
__global__ __launch_bounds__(WAVES * 64, 2) void cross_fwd_kernel(CrossArgs a) {
    constexpr int TILE = KEYS * D * 2, SLOT = 2 * TILE, COPIES = TILE / 1024 / 4;
    constexpr int Q_AT = WAVES == 8 ? 2 * SLOT : SLOT, K_FIRST = WAVES == 8 ? 2 * SLOT + 8 * ROWS32<D> : 2 * SLOT;
    extern __shared__ __attribute__((aligned(16))) uint8_t smem[];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), half = lane >> 5, l32 = lane & 31;
    const int head = blockIdx.x % a.nkv, dh = a.d;
    const Item it = find_item(a, blockIdx.x / a.nkv, WAVES * 32, 0);
    const Group g(a);
    const Rows mine(it, g, it.index * WAVES * 32 + wave * 32);
    const int kbeg = it.lo, kend = it.hi;
    const bf16_t *const K = (const bf16_t *)a.k + (long)head * dh, *const V = (const bf16_t *)a.v + (long)head * dh;

    bf16x8 qf[KS];
    f32x16 oacc[CB];
#pragma unroll
    for (int c = 0; c < CB; ++c) oacc[c] = zero16();
    float m_run = -INFINITY, msc = 0.f, l_run = 0.f;    // reference of the exponentials (raw score), in the exponent's units, row sum
    const float sl2 = a.scale * LOG2E;

    RowCopier<D, COPIES> cpk, cpv;
    cpk.init((wave & 3) * COPIES, a.ldk, dh);
    cpv.init((wave & 3) * COPIES, a.ldv, dh);
    auto copy_kv = [&](uint8_t *slot, int kt) {
        if (WAVES == 4 || wave >= 4) cpk.issue(rows_rsrc(K, kt + 32, a.ldk, kend - kt - 32, dh), slot, 0, 0, 0);
        if (WAVES == 4 || wave < 4) cpv.issue(rows_rsrc(V, kt, a.ldv, kend - kt, dh), slot + TILE, 0, 0, 0);
    };
    uint8_t *const st_q = smem + Q_AT + wave * ROWS32<D>;
    copy_rows<D>((const bf16_t *)a.q + (long)head * g.n * dh, a.ldq, dh, mine, g, st_q);
    if (wave >= WAVES - 4 && wave < WAVES - 2) cpk.issue(rows_rsrc(K, kbeg, a.ldk, kend - kbeg, dh), smem + K_FIRST, 0, 0, 0);
    copy_kv(smem, kbeg);
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) qf[ks] = frag_k<D>(st_q, l32, ks, half);

    TrReader<D> tr;
    const uint32_t lds0 = (uint32_t)(uintptr_t)(lds_void *)smem;
    tr.init(lds0);
    uint32_t kadr[KS];
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) kadr[ks] = lds0 + (l32 * (D / 8) + ((2 * ks + half) ^ swz_unit<D>(l32))) * 16;
    f32x16 s[2];                                         // scores of the blocks of either parity
    uint32_t pp[8];
    // element i of a block: its exponential, the row sum, packed in pairs.  Register i  <->  key kb + 8 (i >> 2) + 4 half + (i & 3)
    auto element = [&](auto I_, const f32x16 &cur, float &keep) {
        constexpr int i = decltype(I_)::value;
        const float p = __builtin_amdgcn_exp2f(fmaf(cur[i], sl2, -msc));
        l_run += p;
        asm volatile("" : "+v"(l_run));
        if constexpr (i & 1) pp[i >> 1] = pack_bf16x2(keep, p);
        else keep = p;
    };
    auto p_frag = [&](auto M_) {
        constexpr int m = decltype(M_)::value;
        const rawx4 w = {pp[4 * m], pp[4 * m + 1], pp[4 * m + 2], pp[4 * m + 3]};
        return *reinterpret_cast<const bf16x8 *>(&w);
    };
    auto mask = [&](f32x16 &x, int kb) {
        const int left = kend - kb - 4 * half;
#pragma unroll
        for (int i = 0; i < 16; ++i) x[i] = 8 * (i >> 2) + (i & 3) < left ? x[i] : -INFINITY;
    };
    auto max16 = [&](const f32x16 &x) {
        float mx = x[0];
#pragma unroll
        for (int i = 1; i < 16; ++i) mx = fmaxf(mx, x[i]);
        return mx;
    };
    float m_limit = -INFINITY;                           // the maximum that moves the reference
    const float lazy = LAZY_LOG2 / sl2;
    auto follow = [&](float mx, auto STRICT_) {
        if (__builtin_amdgcn_ballot_w64(mx > m_limit) == 0) return;
        mx = max_across_halves(mx);
        const bool need = mx > m_limit;
        const float corr = need ? __builtin_amdgcn_exp2f((m_run - mx) * sl2) : 1.f;
        m_run = need ? mx : m_run;
        m_limit = decltype(STRICT_)::value ? m_run : m_run + lazy;
        msc = m_run == -INFINITY ? 0.f : m_run * sl2;
        l_run *= corr;
#pragma unroll
        for (int c = 0; c < CB; ++c)
#pragma unroll
            for (int i = 0; i < 16; ++i) oacc[c][i] *= corr;
    };
    // block b of a step, whose scores are in s[b]: its exponentials and products with V, and the scores of the block behind it (keys nb ..)
    auto block = [&](auto SLOT_, auto B_, int nb) {
        constexpr int b = decltype(B_)::value, NI = KS + 2 * CB, AHEAD = 4, AT = decltype(SLOT_)::value * SLOT;
        const f32x16 &cur = s[b];
        f32x16 &nxt = s[b ^ 1];
        bf16x8 fr[KS];
        shortx4 v0[2 * CB], v1[2 * CB];
        auto issue = [&](auto X_) {
            constexpr int x = decltype(X_)::value;
            if constexpr (x < KS) lds_read16<AT + b * 64 * D>(fr[x], kadr[x]);
            else if constexpr (x < NI) {
                constexpr int m = (x - KS) / CB, c = (x - KS) % CB;
                v0[x - KS] = TrReader<D>::template read_at<b, m, c, 0, AT + TILE>(tr.off);
                v1[x - KS] = TrReader<D>::template read_at<b, m, c, 1, AT + TILE>(tr.off);
            }
        };
        float keep = 0.f, mx = -INFINITY;
        static_for<0, AHEAD>([&](auto X_) { issue(X_); });
        __builtin_amdgcn_sched_barrier(0);
        constexpr int E0 = 2, SPAN = KS + CB;
        static_for<0, E0>([&](auto I_) { element(I_, cur, keep); });
        __builtin_amdgcn_sched_barrier(0);
        static_for<0, NI>([&](auto X_) {
            constexpr int x = decltype(X_)::value;
            constexpr int behind = lds_ops<KS, NI>(x + 1, x + AHEAD);       // reads issued behind item x's
            if constexpr (x < KS) {
                asm volatile("s_waitcnt lgkmcnt(%1)" : "+v"(fr[x]) : "n"(behind));
                if constexpr (x == 0) nxt = MFMA(fr[x], qf[x], zero16());
                else nxt = MFMA(fr[x], qf[x], nxt);
            } else {
                constexpr int m = (x - KS) / CB, c = (x - KS) % CB;
                asm volatile("s_waitcnt lgkmcnt(%2)" : "+v"(v0[x - KS]), "+v"(v1[x - KS]) : "n"(behind));
                oacc[c] = MFMA(join(v0[x - KS], v1[x - KS]), p_frag(std::integral_constant<int, m>{}), oacc[c]);
            }
            issue(std::integral_constant<int, x + AHEAD>{});
            constexpr int lo = x < SPAN ? E0 + (16 - E0) * x / SPAN : 16, hi = x + 1 < SPAN ? E0 + (16 - E0) * (x + 1) / SPAN : 16;
            static_for<lo, hi>([&](auto I_) { element(I_, cur, keep); });
            if constexpr (x > KS) {
                constexpr int d0 = 16 * (x - KS - 1) / (2 * CB - 1), d1 = 16 * (x - KS) / (2 * CB - 1);
                static_for<d0, d1>([&](auto I_) { mx = fmaxf(mx, nxt[decltype(I_)::value]); });
                asm volatile("" : "+v"(mx));
            }
            __builtin_amdgcn_sched_barrier(0);
        });
        if (nb + 32 > kend) {
            mask(nxt, nb);
            mx = max16(nxt);
        }
        follow(mx, std::false_type{});
    };
    const bool live = mine.left > 0;                     // (a wavefront behind a run's last row copies its share, and leaves the units to others)
    auto step = [&](auto SLOT_, int kt) {
        constexpr int slot = decltype(SLOT_)::value;
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");             // this step's tiles have landed
        lds_barrier();                                               // ... and everyone is done with the other slot
        if (kt == kbeg && live) {
            f32x16 x = zero16();
#pragma unroll
            for (int ks = 0; ks < KS; ++ks) x = MFMA(lds_load<bf16x8>(kadr[ks] + K_FIRST), qf[ks], x);
            if (kbeg + 32 > kend) mask(x, kbeg);
            s[0] = x;
            follow(max16(x), std::true_type{});
        }
        if (live) block(SLOT_, std::integral_constant<int, 0>{}, kt + 32);
        // (behind the first block: right behind the barrier all wavefronts would wait for each other at the copies)
        if (kt + KEYS < kend) copy_kv(smem + (slot ^ 1) * SLOT, kt + KEYS);
        if (kt + 32 < kend && live) block(SLOT_, std::integral_constant<int, 1>{}, kt + KEYS);
    };
    for (int kt = kbeg; kt < kend; kt += 2 * KEYS) {
        step(std::integral_constant<int, 0>{}, kt);
        if (kt + KEYS >= kend) break;
        step(std::integral_constant<int, 1>{}, kt + KEYS);
    }

    lds_barrier();                                       // the tiles are done with: LDS now stages the output rows
    const float l_tot = sum_across_halves(l_run);
    store_rows_at<D, CB>(smem + wave * STAGE<D>, oacc, l_tot > 0.f ? 1.f / l_tot : 0.f, (bf16_t *)a.o + (long)head * g.n * dh, a.ldo, dh, mine, g);
    if (a.lse && half == 0 && l32 < mine.left) {
        const int tok = g.token(mine.j + l32), h = head * g.n + mine.j + l32 - tok * g.n;
        a.lse[(long)h * a.Tq + mine.t + tok] = natural_lse(m_run, l_tot, sl2);
    }
}

// ---- forward, few rows ----------------------------------------------------------------------------------------------------
// Up to 32 rows per workgroup, whose wavefronts (eight with 64-wide heads, four with wider ones; two or one where there are many workgroups) share out the blocks of 32 keys, each with two LDS slots of its
// own and no barrier on the way: the next block is in flight while one is multiplied.  Three tokens of 16 heads of 64, 577 keys each: 6.7 us, 8.6 with four
// wavefronts and four slots.  16 tokens of 64 heads of 128, on 8, each over 6144 keys: 80 us, 5.1 TB/s of keys and values, which is what bounds it.  Where that leaves the chip empty or one workgroup with a long walk, the keys are cut into chunks, one per workgroup, whose partial
// results (32 rows of fp32, maximum and sum) cross_combine_kernel joins.
constexpr int FEW_SLOTS = 2;
template <int D> constexpr int FEW_WAVES = D <= 64 ? 8 : 4;
template <int D, int NW> constexpr int FEW_LDS = NW * FEW_SLOTS * 2 * ROWS32<D>;

template <int D, int KS, int CB, int NW>
__global__ __launch_bounds__(64 * NW, 1) void cross_fwd_few_kernel(CrossArgs a) {
    constexpr int N = ROWS32<D> / 1024, SLOT = 2 * ROWS32<D>, SLOTS = FEW_SLOTS, MINE = SLOTS * SLOT, NEXT = 32 * NW;
    extern __shared__ __attribute__((aligned(16))) uint8_t smem_all[];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), half = lane >> 5, l32 = lane & 31;
    uint8_t *const smem = smem_all + wave * MINE;
    const int head = blockIdx.x % a.nkv, dh = a.d;
    const Item it = find_item(a, blockIdx.x / a.nkv, FEW_ROWS, a.chunk);
    const int parts = a.chunk ? max((it.hi - it.lo + a.chunk - 1) / a.chunk, 1) : 1;
    const Group g(a);
    const Rows mine(it, g, it.index / parts * FEW_ROWS);
    const int kbeg = it.lo + it.index % parts * a.chunk, kend = parts > 1 ? min(kbeg + a.chunk, it.hi) : it.hi;
    const bf16_t *const K = (const bf16_t *)a.k + (long)head * dh, *const V = (const bf16_t *)a.v + (long)head * dh;
    const float sl2 = a.scale * LOG2E;

    RowCopier<D, N> cpk, cpv;
    cpk.init(0, a.ldk, dh);
    cpv.init(0, a.ldv, dh);
    auto copy_kv = [&](uint8_t *slot, int kb) {
        cpk.issue(rows_rsrc(K, kb, a.ldk, min(kend - kb, 32), dh), slot, 0, 0, 0);
        cpv.issue(rows_rsrc(V, kb, a.ldv, min(kend - kb, 32), dh), slot + ROWS32<D>, 0, 0, 0);
    };
    // SLOTS - 1 blocks are on their way at any time; what stands behind the last key is copied as zeros, so that a wait counts the same everywhere
    int kb = kbeg + 32 * wave;
    copy_rows<D>((const bf16_t *)a.q + (long)head * g.n * dh, a.ldq, dh, mine, g, smem + (SLOTS - 1) * SLOT);
    static_for<0, SLOTS - 1>([&](auto S_) { copy_kv(smem + decltype(S_)::value * SLOT, kb + NEXT * decltype(S_)::value); });
    asm volatile("s_waitcnt vmcnt(%0)" ::"n"(2 * N * (SLOTS - 1)) : "memory");
    const uint32_t lds0 = (uint32_t)(uintptr_t)(lds_void *)smem;
    uint32_t kadr[KS];
    bf16x8 qf[KS];
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) kadr[ks] = lds0 + (l32 * (D / 8) + ((2 * ks + half) ^ swz_unit<D>(l32))) * 16;
    static_for<0, KS>([&](auto K_) { lds_read16<(SLOTS - 1) * SLOT>(qf[decltype(K_)::value], kadr[decltype(K_)::value]); });
    static_for<0, KS>([&](auto K_) { lds_wait<0>(qf[decltype(K_)::value]); });
    TrReader<D> tr;
    tr.init(lds0);
    f32x16 oacc[CB];
#pragma unroll
    for (int c = 0; c < CB; ++c) oacc[c] = zero16();
    float m_run = -INFINITY, l_run = 0.f;
    auto block = [&](auto SLOT_, int kb) {
        constexpr int AT = decltype(SLOT_)::value * SLOT;
        bf16x8 fr[KS];
        shortx4 v0[2 * CB], v1[2 * CB];
        static_for<0, KS>([&](auto K_) { lds_read16<AT>(fr[decltype(K_)::value], kadr[decltype(K_)::value]); });
        f32x16 s = zero16();
        static_for<0, KS>([&](auto K_) {
            constexpr int ks = decltype(K_)::value;
            lds_wait<KS - 1 - ks>(fr[ks]);
            s = MFMA(fr[ks], qf[ks], s);
        });
        static_for<0, 2 * CB>([&](auto X_) {
            constexpr int x = decltype(X_)::value;
            v0[x] = TrReader<D>::template read_at<0, x / CB, x % CB, 0, AT + ROWS32<D>>(tr.off);
            v1[x] = TrReader<D>::template read_at<0, x / CB, x % CB, 1, AT + ROWS32<D>>(tr.off);
        });
        if (kb + 32 > kend) {
            const int left = kend - kb - 4 * half;
#pragma unroll
            for (int i = 0; i < 16; ++i) s[i] = 8 * (i >> 2) + (i & 3) < left ? s[i] : -INFINITY;
        }
        float mx = s[0];
#pragma unroll
        for (int i = 1; i < 16; ++i) mx = fmaxf(mx, s[i]);
        mx = max_across_halves(mx);
        const bool need = (mx - m_run) * sl2 > LAZY_LOG2;
        if (__builtin_amdgcn_ballot_w64(need) != 0) {
            const float corr = need ? __builtin_amdgcn_exp2f((m_run - mx) * sl2) : 1.f;
            m_run = need ? mx : m_run;
            l_run *= corr;
#pragma unroll
            for (int c = 0; c < CB; ++c)
#pragma unroll
                for (int i = 0; i < 16; ++i) oacc[c][i] *= corr;
        }
        const float msc = m_run == -INFINITY ? 0.f : m_run * sl2;
        float p[16];
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            p[i] = __builtin_amdgcn_exp2f(fmaf(s[i], sl2, -msc));
            l_run += p[i];
        }
        const bf16x8 pf[2] = {pack8(p), pack8(p + 8)};
        static_for<0, 2 * CB>([&](auto X_) {
            lds_wait<0>(v0[decltype(X_)::value]);
            lds_wait<0>(v1[decltype(X_)::value]);
        });
        static_for<0, 2 * CB>([&](auto X_) {
            constexpr int x = decltype(X_)::value;
            oacc[x % CB] = MFMA(join(v0[x], v1[x]), pf[x / CB], oacc[x % CB]);
        });
    };
    while (kb < kend)
        static_for<0, SLOTS>([&](auto S_) {
            constexpr int slot = decltype(S_)::value;
            if (kb >= kend) return;
            asm volatile("" ::: "memory");               // (the slot in front has been read: its reads have been waited for)
            copy_kv(smem + (slot + SLOTS - 1) % SLOTS * SLOT, kb + NEXT * (SLOTS - 1));
            asm volatile("s_waitcnt vmcnt(%0)" ::"n"(2 * N * (SLOTS - 1)) : "memory");
            block(S_, kb);
            kb += NEXT;
        });
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    // the wavefronts' partial softmaxes over disjoint keys become one: each joins blocks of 32 features
    put_acc(smem, oacc);
    const float l_own = sum_across_halves(l_run);
    float2 *const ml = reinterpret_cast<float2 *>(smem + SLOT);
    if (half == 0) ml[l32] = make_float2(m_run, l_own);
    lds_barrier();
    float m = -INFINITY, l = 0.f, mw[NW], f[NW];
#pragma unroll
    for (int w = 0; w < NW; ++w) {
        const float2 v = reinterpret_cast<const float2 *>(smem_all + w * MINE + SLOT)[l32];
        mw[w] = v.x; f[w] = v.y;
        m = fmaxf(m, v.x);
    }
#pragma unroll
    for (int w = 0; w < NW; ++w) {
        const float e = mw[w] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((mw[w] - m) * sl2);
        l += f[w] * e;
        f[w] = e;
    }
    const int tok = g.token(mine.j + l32), h = mine.j + l32 - tok * g.n;
    const bool live = l32 < mine.left;
#pragma unroll
    for (int cb = 0; cb < CB; ++cb) {
        if (cb % NW != wave) continue;
        f32x4 x[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            x[i] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int w = 0; w < NW; ++w) x[i] += reinterpret_cast<const f32x4 *>(smem_all + w * MINE)[(4 * cb + i) * 64 + lane] * f[w];
        }
        const int c0 = 32 * cb + 4 * half;
        if (parts > 1) {
            float *out = a.part + ((size_t)blockIdx.x * FEW_ROWS + l32) * dh + c0;
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (live && c0 + 8 * i < dh) *reinterpret_cast<f32x4 *>(out + 8 * i) = x[i];
        } else {
            const float r = l > 0.f ? 1.f / l : 0.f;
            bf16_t *out = (bf16_t *)a.o + (mine.t + tok) * a.ldo + (long)(head * g.n + h) * dh + c0;
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (live && c0 + 8 * i < dh)
                    *reinterpret_cast<uint2 *>(out + 8 * i) = make_uint2(pack_bf16x2(x[i][0] * r, x[i][1] * r), pack_bf16x2(x[i][2] * r, x[i][3] * r));
        }
    }
    if (wave == NW - 1 && half == 0 && live) {
        if (parts > 1) a.part_ml[(size_t)blockIdx.x * FEW_ROWS + l32] = make_float2(m, l);
        else if (a.lse) a.lse[(long)(head * g.n + h) * a.Tq + mine.t + tok] = natural_lse(m, l, sl2);
    }
}

// The chunks' results of up to 32 rows; a workgroup for each of the kernel's above, of which the one of a chunk 0 does it
__global__ __launch_bounds__(256) void cross_combine_kernel(CrossArgs a) {
    const int head = blockIdx.x % a.nkv, dh = a.d;
    const Item it = find_item(a, blockIdx.x / a.nkv, FEW_ROWS, a.chunk);
    const int parts = max((it.hi - it.lo + a.chunk - 1) / a.chunk, 1);
    if (parts == 1 || it.index % parts) return;
    const Group g(a);
    const Rows mine(it, g, it.index / parts * FEW_ROWS);
    const float sl2 = a.scale * LOG2E;
    const int quads = dh / 4, rows = min(mine.left, FEW_ROWS);
    const size_t stride = (size_t)a.nkv * FEW_ROWS;
    for (int e = threadIdx.x; e < rows * quads; e += 256) {
        const int r = e / quads, c = e % quads * 4;
        const float2 *ml = a.part_ml + (size_t)blockIdx.x * FEW_ROWS + r;
        const float *part = a.part + ((size_t)blockIdx.x * FEW_ROWS + r) * dh + c;
        float m = -INFINITY, l = 0.f;
        f32x4 x = {0.f, 0.f, 0.f, 0.f};
        for (int j0 = 0; j0 < parts; j0 += 8) {        // eight at a time on their way (one by one, and twice over, 8 chunks took 13.5 us; so 5)
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
            const float base = top == -INFINITY ? 0.f : top, corr = __builtin_amdgcn_exp2f((m - base) * sl2);
            l *= corr;
            x *= corr;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float w = __builtin_amdgcn_exp2f((v[i].x - base) * sl2);
                l += v[i].y * w;
                x += y[i] * w;
            }
            m = top;
        }
        const int tok = g.token(mine.j + r), h = head * g.n + mine.j + r - tok * g.n;
        const float f = l > 0.f ? 1.f / l : 0.f;
        *reinterpret_cast<uint2 *>((bf16_t *)a.o + (mine.t + tok) * a.ldo + (long)h * dh + c) =
            make_uint2(pack_bf16x2(x[0] * f, x[1] * f), pack_bf16x2(x[2] * f, x[3] * f));
        if (a.lse && c == 0) a.lse[(long)h * a.Tq + mine.t + tok] = natural_lse(m, l, sl2);
    }
}

template <int D, int KS, int CB, int WAVES>
hipError_t launch_tiles(const CrossArgs &a, int items, hipStream_t st) {
    static std::atomic<bool> done{false};
    constexpr int LDS = std::max(FWD_LDS<D, WAVES>, WAVES * STAGE<D>);
    const hipError_t e = set_smem(done, cross_fwd_kernel<D, KS, CB, WAVES>, LDS);
    if (e != hipSuccess) return e;
    cross_fwd_kernel<D, KS, CB, WAVES><<<items * a.nkv, WAVES * 64, LDS, st>>>(a);
    return hipGetLastError();
}

template <int D, int KS, int CB, int NW>
hipError_t launch_few(const CrossArgs &a, int items, hipStream_t st) {
    static std::atomic<bool> done{false};
    const hipError_t e = set_smem(done, cross_fwd_few_kernel<D, KS, CB, NW>, FEW_LDS<D, NW>);
    if (e != hipSuccess) return e;
    cross_fwd_few_kernel<D, KS, CB, NW><<<items * a.nkv, 64 * NW, FEW_LDS<D, NW>, st>>>(a);
    if (a.chunk) cross_combine_kernel<<<items * a.nkv, 256, 0, st>>>(a);
    return hipGetLastError();
}

template <int D, int KS, int CB>
hipError_t launch_fwd(const CrossArgs &a, const CrossPlan &p, hipStream_t st) {
    if (p.rows == FEW_ROWS)
        return p.waves == 1 ? launch_few<D, KS, CB, 1>(a, p.items, st) : p.waves == 2 ? launch_few<D, KS, CB, 2>(a, p.items, st)
                                                                                       : launch_few<D, KS, CB, FEW_WAVES<D>>(a, p.items, st);
    return p.rows == 256 ? launch_tiles<D, KS, CB, 8>(a, p.items, st) : launch_tiles<D, KS, CB, 4>(a, p.items, st);
}

}  // namespace

hipError_t cross_mfma_fwd(const CrossArgs &a, const CrossPlan &p, hipStream_t st) {
    return a.d <= 64 ? launch_fwd<64, 4, 2>(a, p, st) : a.d <= 80 ? launch_fwd<128, 5, 3>(a, p, st) : a.d <= 96 ? launch_fwd<128, 6, 3>(a, p, st)
                                                                                                          : launch_fwd<128, 8, 4>(a, p, st);
}

}  // namespace mmt
