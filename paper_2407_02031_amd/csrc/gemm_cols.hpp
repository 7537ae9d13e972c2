// Products of rows, D[m][n] = sum_k P[m][k] Q[n][k], both operands in bf16 or both in 8 bits with scales (fp8.hpp), for epilogues that need several columns of a row in one lane: a gate
// beside its value, a block's largest element.
//
// Tiling and loads as in gemm_tile.hpp: BM x BN tiles of WGM x WGN wavefronts, operands straight into LDS in steps of 128 bytes of K, a ring of STAGES such steps, 16-byte chunks swizzled.
// What differs:
//   - A step is 64 elements of bf16, two MFMAs 16x16x32 deep, or 128 of 8 bits, one scaled MFMA 16x16x128.  The scales of a step's rows ride along in LDS, a byte a row, and the
//     MFMA multiplies by them: both operands' blocks are 128 long, so all four 32-element pieces of a lane's row have the same one.
//   - The 16 rows of an MFMA operand are not neighbours: of 32 (64) rows of Q, block b takes every second (fourth), so that a lane, which holds elements 4 quad .. 4 quad + 3 of
//     each block's result, has 8 (16) neighbouring columns of one row of D in all.  Epilogues work in registers and store 16 bytes a lane, without a detour through LDS.  The
//     rows are sorted where they are loaded: which row of memory goes into which row of LDS costs nothing.  The same for P, four blocks to 64 rows, whose four scales are then one word.
//   - Gated: half of a wavefront's Q blocks are rows of the value, half rows of the gate, of the same columns.
//   - KS = 2: WGM x WGN wavefronts work on the first half of each step, as many on the second, and their sums meet in LDS.  A wavefront alone on its SIMD issues a vector instruction every
//     3.1 to 4 ns, two together one every 2: so in tiles that would have four wavefronts on a CU, mostly those of widened operands (1976 x 1280 x 5120 onto fp32 41 -> 35 us with 96 x 128) and of
//     long reductions (gated in bf16, 512 x 640 x 2560 14.4 -> 12.9 with 64 x 64, 1024 x 1280 x 5120 65 -> 53 with 128 x 128).
#pragma once
#include "gemm_dma.hpp"
#include "cols_index.hpp"
#include "fp8.hpp"

namespace sd {

typedef int i32x8 __attribute__((ext_vector_type(8)));

struct ColsProblem {
    const uint8_t *p, *q;              // [M, Kb], [N or 2 N, Kb] bytes: values first, then gates
    const uint8_t *ps, *qs;            // scales (8 bits)
    int64_t ldps, ldqs;
    const uint16_t* bias;              // [N or 2 N] or null
    const void* res;                   // [M, N] of y's type or null
    void* y;                           // [M, N]
    uint16_t* z;                       // gated: [M, 2 N] bf16 or null
    uint8_t* ys;                       // y in 8 bits: its scales
    int64_t ldys;
    int32_t M, N, Kb;                  // Kb: bytes of a row of P or Q, a multiple of 16
    int32_t act, y_f32;
    int32_t tiles_m, tiles_n;
};

template <bool FP8, int BM, int BN, int WGN, int STAGES, bool OUT8>
constexpr int cols_lds_chunks() {
    const int ring = STAGES * ColsTileIndex<FP8, BM, BN, 1, 1, 1, STAGES, false, OUT8>::STAGE;
    return ring + BN / 4 + (OUT8 ? WGN * BM / 4 : 0);
}

__device__ __forceinline__ void dma4(const void* gptr, uint32_t lds_base) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, off" ::"s"(__builtin_amdgcn_readfirstlane(lds_base)), "v"(gptr) : "memory", "m0");
}

// What the operands are, and how they are multiplied.  The scaled MFMA takes 128 of 8 bits in the time of 64 of bf16, but it adds products eight at a time, and of those eight it keeps what is worth 2^-13 of
// the largest and more (measured: with one of 2^16, another of 2^2 is gone; in another eight, and of the sums of eights, nothing is): off by 1.5e-5 of a sum of random terms, where
// 8 bits were off by 2^-5 in each.  That is far below the rounding of y to bf16 or to 8 bits, but not of y in fp32: there, where the caller asks for whole sums, and where the rows are few
// and the operands' bytes all that counts, they are widened to bf16, with their scales and exactly (elements from 2^-126 to below 2^128;
// smaller ones to multiples of 2^-133, larger ones to infinities, which the scaled MFMA would multiply), and multiplied as those.
enum ColsMode { COLS_BF16, COLS_FP8, COLS_FP8_WIDE };

// Eight e4m3 elements times 2^(s - 127), s a byte, which is what the conversion looks at of an fp32 scale
__device__ __forceinline__ bf16x8 widen8(uint32_t lo, uint32_t hi, uint32_t s) {
    const float scale = __uint_as_float(s << 23);
    union { bf16x8 v; bf16x2 p[4]; } u;
    u.p[0] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, false);
    u.p[1] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, true);
    u.p[2] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, false);
    u.p[3] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, true);
    return u.v;
}
// ... eight of a lane's 32 of a step
template <int H>
__device__ __forceinline__ bf16x8 widen8(const u32x4 (&w)[H], int i, uint32_t s) { return widen8(w[i / 2][i % 2 * 2], w[i / 2][i % 2 * 2 + 1], s); }
__device__ __forceinline__ void widen32(const u32x4 (&w)[2], uint32_t s, bf16x8 (&o)[4]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) o[i] = widen8(w, i, s);
}
__device__ __forceinline__ f32x4 mfma_bf16(bf16x8 q, bf16x8 p, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(q, p, c, 0, 0, 0); }
__device__ __forceinline__ i32x8 words8(const u32x4 (&w)[2]) {
    return i32x8{(int)w[0][0], (int)w[0][1], (int)w[0][2], (int)w[0][3], (int)w[1][0], (int)w[1][1], (int)w[1][2], (int)w[1][3]};
}
// c + (Q block) (P block)^T, scales bytes QB of qs and PB of ps
template <int QB, int PB>
__device__ __forceinline__ f32x4 mfma_fp8(const u32x4 (&q)[2], const u32x4 (&p)[2], f32x4 c, uint32_t qs, uint32_t ps) {
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(words8(q), words8(p), c, 0, 0, QB, (int)qs, PB, (int)ps);
}
// f(integral_constant<int, 0>) ... f(integral_constant<int, N - 1>)
template <int N, class F, int I = 0>
__device__ __forceinline__ void each(F f) {
    if constexpr (I < N) {
        f(std::integral_constant<int, I>());
        each<N, F, I + 1>(f);
    }
}

template <int MODE, int BM, int BN, int WGM, int WGN, int KS, int STAGES, bool GATED, bool OUT8, bool GUARD>
__device__ __forceinline__ void cols_tile(const ColsProblem& P, const int tile, u32x4* const lds) {
    constexpr bool FP8 = MODE != COLS_BF16, WIDE = MODE == COLS_FP8_WIDE;
    using I = ColsTileIndex<FP8, BM, BN, WGM, WGN, KS, STAGES, GATED, OUT8>;
    constexpr int NW = I::NW, WM = I::WM, WN = I::WN, MI = I::MI, NI = I::NI, LPT = I::LPT, STAGE = I::STAGE, PIECES = I::PIECES, NV = I::NV, BP = I::BP, BQ = I::BQ, BN_OUT = I::BN_OUT, WN_OUT = I::WN_OUT;
    constexpr int HC = 2 / KS;                         // chunks of a row's step that a lane works on
    constexpr int LOADS = LPT + (FP8 ? 1 : 0);
    constexpr int RING = NI >= 4 ? NI / 2 : NI;
    static_assert(MI % BP == 0 && NV % BQ == 0 && NI % RING == 0 && (!WIDE || NI % 2 == 0) && STAGES >= 2 && STAGES <= 4, "tile");
    static_assert(KS == 1 || (KS == 2 && MODE != COLS_FP8 && MI % 2 == 0 && WGM * WGN * MI * NI * 64 <= STAGES * STAGE), "halves");
    static_assert(!FP8 || PIECES <= NW, "scales");
    static_assert(NW * 64 >= BN, "bias");
    static_assert(!OUT8 || (GATED && FP8 && BN_OUT == FP8_BLOCK), "a tile's columns are one block of y");

    const int band_tiles = 8 * P.tiles_n;
    const int band = tile / band_tiles, rem = tile - band * band_tiles;
    const int band_rows = min(8, P.tiles_m - band * 8);
    const int tn = rem / band_rows, tm = band * 8 + rem % band_rows;
    const int m0 = tm * BM, n0 = tn * BN_OUT;
    const int M = P.M, N = P.N, Kb = P.Kb;
    const int nk = (Kb + 127) / 128;

    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int l16 = lane & 15, quad = lane >> 4;
    const int half = KS == 2 ? wave / (WGM * WGN) : 0;
    const int wm = (KS == 2 ? wave % (WGM * WGN) : wave) / WGN * WM, wn = (wave % WGN) * WN, wn_out = (wave % WGN) * WN_OUT;

    // ---- loads (cols_index.hpp).  They lie in one block, so what differs between value and gate is the wavefront's base.
    uint32_t off[LPT];
    const uint8_t* base[LPT];
    const uint8_t* const pb = P.p + (int64_t)m0 * Kb;
    const uint8_t* const qb = P.q + (int64_t)n0 * Kb;
    auto chunk = [&](int j) { return I::chunk(I::eight(j, wave), lane); };
#pragma unroll
    for (int j = 0; j < LPT; ++j) {
        const int first = I::eight(j, wave) * 8, row = first + (lane >> 3);
        if (I::of_p(j, first)) {
            base[j] = pb;
            off[j] = (uint32_t)I::p_row(first, row, m0, M) * (uint32_t)Kb + chunk(j) * 16;
        } else {
            base[j] = I::q_gate(first) ? qb + (int64_t)N * Kb : qb;
            off[j] = (uint32_t)I::q_row(first, row, n0, N) * (uint32_t)Kb + chunk(j) * 16;
        }
    }
    // what the epilogue adds to columns: thread j has that of the tile's j-th (of the value's, then of the gate's)
    uint16_t bias_raw = 0;
    if (P.bias && tid < BN) {
        const int j = GATED && tid >= BN_OUT ? tid - BN_OUT : tid;
        if (n0 + j < N) bias_raw = P.bias[n0 + j + (GATED && tid >= BN_OUT ? N : 0)];
    }
    const uint8_t* sp = nullptr;
    int64_t sp_step = 0;
    if constexpr (FP8) {
        const int a = (wave % PIECES) * 64 + lane;
        if (I::scale_of_p(a)) {
            sp = P.ps + I::p_scale(a, m0, M);
            sp_step = P.ldps;
        } else {
            sp = P.qs + I::q_scale(a, n0, N);
            sp_step = P.ldqs;
        }
    }
    const uint32_t lds_base = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) void*)lds;
    const uint32_t scale_base = lds_base + (uint32_t)((BM + BN) * 128 + (PIECES ? wave % (PIECES ? PIECES : 1) : 0) * 256);
    // load j of step t; steps are loaded in order, each once
    auto load = [&](int j, int t, int stg, auto partial) {
        const uint32_t to = lds_base + (uint32_t)stg * (STAGE * 16) + (uint32_t)I::eight(j, wave) * 1024;
        const int kb = t * 128;
        if (decltype(partial)::value && kb + 128 > Kb) {
            const uint8_t* const src = base[j] + kb + off[j];
            dma16(I::there(kb, chunk(j), Kb) ? src : reinterpret_cast<const uint8_t*>(g_gemm_zeros), to);
        } else {
            dma16_so(base[j] + kb, off[j], to);
        }
        if (FP8 && j == 0) {
            dma4(sp, scale_base + (uint32_t)stg * (STAGE * 16));
            sp += sp_step;
        }
    };

    f32x4 acc[MI][NI];
#pragma unroll
    for (int mi = 0; mi < MI; ++mi)
#pragma unroll
        for (int ni = 0; ni < NI; ++ni) acc[mi][ni] = f32x4{0.f, 0.f, 0.f, 0.f};

    // ---- operands in registers: P's blocks, and a ring of Q's.  A lane has chunks quad and quad + 4 of a row, of halves the one or the other, of either operand: which k an MFMA's lane has does not matter, if it is the same ones.
    u32x4 pr[MI][HC], qr[RING][HC];
    uint32_t ps[FP8 ? MI / BP : 1], qs[FP8 ? NI / BQ : 1];     // scales of the step being multiplied
    const u32x4* const frag = lds + l16 * 8;
    auto part = [&](int h) { return I::part(l16, (KS == 2 ? half : h) * 4 + quad); };
    auto fetch_p = [&](int st, int mi) {
#pragma unroll
        for (int h = 0; h < HC; ++h) pr[mi][h] = frag[st * STAGE + I::p_block(wm, mi) + part(h)];
    };
    auto fetch_q = [&](int st, int ni) {
#pragma unroll
        for (int h = 0; h < HC; ++h) qr[ni % RING][h] = frag[st * STAGE + I::q_block(wn, ni) + part(h)];
    };
    auto fetch_scales = [&](int st, auto& p, auto& q) {
        if constexpr (FP8) {
            const uint8_t* const sc = reinterpret_cast<const uint8_t*>(lds) + st * (STAGE * 16) + (BM + BN) * 128;
#pragma unroll
            for (int i = 0; i < MI / BP; ++i) {
                const uint8_t* const at = sc + I::p_scales_at(wm, i, l16);
                p[i] = BP == 4 ? *reinterpret_cast<const uint32_t*>(at) : *reinterpret_cast<const uint16_t*>(at);
            }
#pragma unroll
            for (int i = 0; i < NI / BQ; ++i) {
                const uint8_t* const at = sc + I::q_scales_at(wn_out, i, l16);
                q[i] = BQ == 4 ? *reinterpret_cast<const uint32_t*>(at) : *reinterpret_cast<const uint16_t*>(at);
            }
        }
    };
    uint32_t ps_next[FP8 ? MI / BP : 1], qs_next[FP8 ? NI / BQ : 1];
    // Widened: all of P's blocks, and Q's block of this slot and the next
    bf16x8 pw[WIDE ? MI : 1][2 * HC], qw[2][2 * HC];
    auto scale_of = [](auto& words, int i, auto per) { return (words[i / decltype(per)::value] >> (i % decltype(per)::value * 8)) & 255u; };
    using PerP = std::integral_constant<int, BP>;
    using PerQ = std::integral_constant<int, BQ>;
    // Slot s: Q block s by all of P's, then `load`'s share of another step's loads, dealt over the slots from the edge on.  (No branches in here: the compiler would move the MFMAs past them, all
    // to the end of the step.)
    auto slot = [&](auto sc, auto refill_qc, auto refill_pc, int st_q, auto load) {
        constexpr int s = decltype(sc)::value;
        constexpr bool refill_q = decltype(refill_qc)::value, refill_p = decltype(refill_pc)::value;
        __builtin_amdgcn_sched_barrier(0);
        if constexpr (WIDE) {
            // What the slot multiplies was widened in the one before; in the last, P's blocks of the next step are, behind the products.  Raw blocks are free a slot earlier than they would be,
            // and the compiler may order the slot's conversions and products (put between them one by one they took 15 % longer).
            constexpr bool last = s == NI - 1;
            if constexpr (refill_p)
#pragma unroll
                for (int mi = 0; mi < MI; ++mi) fetch_p(st_q, mi);
            if constexpr (refill_q) fetch_q(st_q, (s + RING) % NI);
#pragma unroll
            for (int i = 0; i < 2 * HC; ++i)
                if constexpr (!last) qw[(s + 1) % 2][i] = widen8(qr[(s + 1) % RING], i, scale_of(qs, s + 1, PerQ()));
#pragma unroll
            for (int i = 0; i < 2 * HC; ++i)
#pragma unroll
                for (int mi = 0; mi < MI; ++mi) acc[mi][s] = mfma_bf16(qw[s % 2][i], pw[mi][i], acc[mi][s]);
            if constexpr (last && refill_q)
#pragma unroll
                for (int i = 0; i < 2 * HC; ++i) {
                    qw[0][i] = widen8(qr[0], i, scale_of(qs_next, 0, PerQ()));
#pragma unroll
                    for (int mi = 0; mi < MI; ++mi) pw[mi][i] = widen8(pr[mi], i, scale_of(ps_next, mi, PerP()));
                }
        } else {
            each<MI>([&](auto mic) {
                constexpr int mi = decltype(mic)::value;
                f32x4& c = acc[mi][s];
                if constexpr (MODE == COLS_FP8) {
                    c = mfma_fp8<s % BQ, mi % BP>(qr[s % RING], pr[mi], c, qs[s / BQ], ps[mi / BP]);
                } else {
#pragma unroll
                    for (int h = 0; h < HC; ++h) c = mfma_bf16(__builtin_bit_cast(bf16x8, qr[s % RING][h]), __builtin_bit_cast(bf16x8, pr[mi][h]), c);
                }
                if constexpr (refill_p) {
                    __builtin_amdgcn_sched_barrier(0);
                    fetch_p(st_q, mi);
                    __builtin_amdgcn_sched_barrier(0);
                }
            });
        }
        __builtin_amdgcn_sched_barrier(0);
        if constexpr (refill_q && !WIDE) fetch_q(st_q, (s + RING) % NI);
        constexpr int i = (s + RING) % NI, DEAL = STAGES > 2 ? NI : RING;
#pragma unroll
        for (int j = i * LPT / DEAL; j < (i + 1) * LPT / DEAL && i < DEAL; ++j) load(j);
    };
    // A step: its first NI - RING slots (`head`), then, when the next step has landed everywhere and this one's stage is free (what is left of it is in registers), the last RING
    // (`edge`), which bring in the next step's first blocks and, P's as they are done with, all of P.
    auto head = [&](int st, auto load) {
        each<NI - RING>([&](auto s) { slot(s, std::true_type(), std::false_type(), st, load); });
    };
    auto edge = [&](int sn, auto load) {
        fetch_scales(sn, ps_next, qs_next);
        each<RING>([&](auto i) {
            constexpr int s = NI - RING + decltype(i)::value;
            slot(std::integral_constant<int, s>(), std::true_type(), std::integral_constant<bool, s == (WIDE ? NI - RING : NI - 1)>(), sn, load);
        });
        if constexpr (FP8) {
#pragma unroll
            for (int i = 0; i < MI / BP; ++i) ps[i] = ps_next[i];
#pragma unroll
            for (int i = 0; i < NI / BQ; ++i) qs[i] = qs_next[i];
        }
    };
    auto none = [](int) {};
    auto wait_steps = [&](int newer) {      // `newer` steps may stay in flight
        if (STAGES >= 4 && newer >= 3) wait_vmcnt<3 * LOADS>();
        else if (STAGES >= 3 && newer >= 2) wait_vmcnt<2 * LOADS>();
        else if (newer >= 1) wait_vmcnt<LOADS>();
        else wait_vmcnt<0>();
    };

#pragma unroll
    for (int d = 0; d < STAGES; ++d)
        if (d < nk)
#pragma unroll
            for (int j = 0; j < LPT; ++j) load(j, d, d, std::integral_constant<bool, GUARD>());
    wait_steps(nk - 1 < STAGES - 1 ? nk - 1 : STAGES - 1);
    __syncthreads();
    fetch_scales(0, ps, qs);
#pragma unroll
    for (int mi = 0; mi < MI; ++mi) fetch_p(0, mi);
#pragma unroll
    for (int s = 0; s < RING; ++s) fetch_q(0, s);
    if constexpr (WIDE) {
#pragma unroll
        for (int i = 0; i < 2 * HC; ++i) {
#pragma unroll
            for (int mi = 0; mi < MI; ++mi) pw[mi][i] = widen8(pr[mi], i, scale_of(ps, mi, PerP()));
            qw[0][i] = widen8(qr[0], i, scale_of(qs, 0, PerQ()));
        }
    }
    head(0, none);
    int st = 0, t = 0;
    const int nfull = GUARD ? Kb / 128 : nk;     // whole steps
#pragma unroll 1
    for (; t + STAGES < nfull; ++t) {
        wait_vmcnt<(STAGES - 2) * LOADS>();
        __syncthreads();
        const int sn = st + 1 == STAGES ? 0 : st + 1;
        auto next = [&](int j) { load(j, t + STAGES, st, std::false_type()); };
        edge(sn, next);
        head(sn, next);
        st = sn;
    }
    // the last steps, which have nothing left to load but one that may be partial
#pragma unroll 1
    for (; t + 1 < nk; ++t) {
        wait_steps(nk - 2 - t < STAGES - 2 ? nk - 2 - t : STAGES - 2);
        __syncthreads();
        const int sn = st + 1 == STAGES ? 0 : st + 1;
        if (t + STAGES < nk)
#pragma unroll
            for (int j = 0; j < LPT; ++j) load(j, t + STAGES, st, std::integral_constant<bool, GUARD>());
        edge(sn, none);
        head(sn, none);
        st = sn;
    }
    each<RING>([&](auto i) { slot(std::integral_constant<int, NI - RING + decltype(i)::value>(), std::false_type(), std::false_type(), 0, none); });

    // the halves' sums, of which each half finishes one half of the rows' blocks
    constexpr int ME = MI / KS;
    if constexpr (KS == 2) {
        __syncthreads();
        f32x4* const swap = reinterpret_cast<f32x4*>(lds) + I::meet(wave % (WGM * WGN), 0, 0, lane);
#pragma unroll
        for (int i = 0; i < ME * NI; ++i) swap[I::meet(0, 1 - half, i, 0)] = half ? acc[i / NI][i % NI] : acc[ME + i / NI][i % NI];
        __syncthreads();
#pragma unroll
        for (int i = 0; i < ME * NI; ++i) acc[i / NI][i % NI] = (half ? acc[ME + i / NI][i % NI] : acc[i / NI][i % NI]) + swap[I::meet(0, half, i, 0)];
    }
    // ---- epilogue.  A lane has rows spread<BP>(mi, l16) of its wavefront's, and of each group of 16 BQ columns the 4 BQ from 4 BQ quad on.
    constexpr int W4 = BQ, NG = NV / BQ;               // pieces of four columns of a lane in a group; groups
    auto column = [&](int g) { return n0 + I::result_column(wn_out, g, quad); };
    auto row_of = [&](int mi) { return I::result_row(wm, KS == 2 ? half * ME + mi : mi, l16); };
    // element x of piece c of group g, of the blocks from `first` on
    auto element = [&](int mi, int first, int g, int c, int x) -> float& { return reinterpret_cast<float(&)[4]>(acc[mi][first + g * BQ + (4 * c + x) % BQ])[(4 * c + x) / BQ]; };
    auto piece = [&](int mi, int first, int g, int c) {
        return f32x4{element(mi, first, g, c, 0), element(mi, first, g, c, 1), element(mi, first, g, c, 2), element(mi, first, g, c, 3)};
    };
    // the tile's bias, which a thread each has had in a register since the start (fetched here it would take a trip to memory, and held by every lane 16 registers)
    float* const bias = reinterpret_cast<float*>(lds + STAGES * STAGE);
    if (tid < BN) bias[tid] = bf16_to_f32(bias_raw);
    __syncthreads();
    // A row's last columns one by one.  What is stored `past` the caches leaves them to the operands.  z, which waits for the backward pass (us, norm, gated layer and linear layer, past / through: 8192 x 1280
    // to 5120 370 / 386, 16384 x 640 to 2560 211 / 247, 8192 x 320 to 1280 57.3 / 56.6; with their backward passes 1092 / 1095, 734 / 736, 177 / 176).  Not y in bf16 or fp32, though a launch alone would gain up to
    // 13 % (8192 x 1280 to 5120 163 / 188 us): the linear layer behind it loses as much (both 288 / 285, 4096 rows 167 / 162).
    auto store = [&](auto* p, int64_t at, int col, const f32x4 (&v)[W4], auto past) {
        using T = std::remove_pointer_t<decltype(p)>;
        if (col + 4 * W4 <= N) {
#pragma unroll
            for (int c = 0; c < W4; c += 2) {
                if constexpr (std::is_same_v<T, float>) {
                    store4(p + at + 4 * c, v[c]);
                    store4(p + at + 4 * c + 4, v[c + 1]);
                } else if constexpr (decltype(past)::value) {
                    bf16x8u o;
#pragma unroll
                    for (int x = 0; x < 8; ++x) o[x] = (__bf16)v[c + x / 4][x % 4];
                    __builtin_nontemporal_store(o, reinterpret_cast<bf16x8u*>(p + at + 4 * c));
                } else {
                    store8(p + at + 4 * c, f32x8{v[c], v[c + 1]});
                }
            }
        } else
#pragma unroll
            for (int x = 0; x < 4 * W4; ++x)
                if (col + x < N) p[at + x] = (T)v[x / 4][x % 4];
    };
    auto add = [&](auto* p, int64_t at, int col, f32x4 (&v)[W4]) {
        if (col + 4 * W4 <= N) {
#pragma unroll
            for (int c = 0; c < W4; c += 2) {
                const f32x8 r = load8(p + at + 4 * c);
                v[c] += r.lo;
                v[c + 1] += r.hi;
            }
        } else
#pragma unroll
            for (int x = 0; x < 4 * W4; ++x)
                if (col + x < N) v[x / 4][x % 4] += (float)p[at + x];
    };
    __bf16* const zb = reinterpret_cast<__bf16*>(P.z);
    float top[OUT8 ? ME : 1];
#pragma unroll
    for (int mi = 0; mi < (OUT8 ? ME : 1); ++mi) top[mi] = 0.f;
#pragma unroll
    for (int gr = 0; gr < NG; ++gr) {
        const int col = column(gr);
        f32x4 bv[W4], bg[W4];
#pragma unroll
        for (int c = 0; c < W4; ++c) {
            bv[c] = *reinterpret_cast<const f32x4*>(bias + col - n0 + 4 * c);
            if (GATED) bg[c] = *reinterpret_cast<const f32x4*>(bias + BN_OUT + col - n0 + 4 * c);
        }
#pragma unroll
        for (int mi = 0; mi < ME; ++mi) {
            const int m = m0 + row_of(mi);
            f32x4 v[W4], g[W4];
#pragma unroll
            for (int c = 0; c < W4; ++c) {
                v[c] = piece(mi, 0, gr, c) + bv[c];
                if (GATED) g[c] = piece(mi, GATED ? NV : 0, gr, c) + bg[c];
            }
            if constexpr (GATED) {
                if (!OUT8 && P.z && m < M) {
                    store(zb, (int64_t)m * 2 * N + col, col, v, std::true_type());
                    store(zb, (int64_t)m * 2 * N + N + col, col, g, std::true_type());
                }
                apply_act(P.act, g);
#pragma unroll
                for (int c = 0; c < W4; ++c) v[c] *= g[c];
            } else {
                apply_act(P.act, v);
                if (P.res && m < M) {
                    if (P.y_f32) add(static_cast<const float*>(P.res), (int64_t)m * N + col, col, v);
                    else add(static_cast<const __bf16*>(P.res), (int64_t)m * N + col, col, v);
                }
            }
            if constexpr (OUT8) {
                // kept where the value's sums were, until the block's largest is known (N is a multiple of 16: a lane's columns are all there or none)
#pragma unroll
                for (int c = 0; c < W4; ++c) {
                    if (col < N) top[mi] = fp8_top(top[mi], v[c]);
#pragma unroll
                    for (int x = 0; x < 4; ++x) element(mi, 0, gr, c, x) = v[c][x];
                }
            } else if (m < M) {
                if (P.y_f32) store(static_cast<float*>(P.y), (int64_t)m * N + col, col, v, std::false_type());
                else store(static_cast<__bf16*>(P.y), (int64_t)m * N + col, col, v, std::false_type());
            }
        }
    }
    if constexpr (OUT8) {
        uint32_t* const meet = reinterpret_cast<uint32_t*>(bias + BN);      // [WGN][BM]
        bool finite = true;
#pragma unroll
        for (int mi = 0; mi < ME; ++mi) {
            uint32_t u = __float_as_uint(top[mi]);
            if (u >= 0x7f800000u) {
                finite = false;
                u = 0;
#pragma unroll
                for (int i = 0; i < NG * W4; ++i)
                    if (column(i / W4) < N) u = fp8_magnitude(u, piece(mi, 0, i / W4, i % W4));
            }
            u = max(u, (uint32_t)__shfl_xor((int)u, 16));
            u = max(u, (uint32_t)__shfl_xor((int)u, 32));
            if (quad == 0) meet[(wave % WGN) * BM + row_of(mi)] = u;
        }
        __syncthreads();
        const bool plain = __all(finite);
        // (y of half the bytes, if it is large, does: 8192 x 1280 to 5120 92.3 / 104.7 us past / through, with the linear layer behind it 213 / 218, 4096 rows 54 / 63.5 and 115.4 / 116.8; 1024 rows 25.4 / 27.7, but 51.2 / 49.7)
        const bool past = (int64_t)M * N > 8ll << 20;
#pragma unroll
        for (int mi = 0; mi < ME; ++mi) {
            const int r = row_of(mi), m = m0 + r;
            uint32_t u = 0;
#pragma unroll
            for (int w = 0; w < WGN; ++w) u = max(u, meet[w * BM + r]);
            const int sc = fp8_scale(u);
            const float inv = fp8_inverse(sc);
            if (m < M) {
                if (wave % WGN == 0 && quad == 0) P.ys[(int64_t)tn * P.ldys + m] = (uint8_t)sc;
#pragma unroll
                for (int g = 0; g < NG; ++g) {
                    u32x4 w;
                    if (plain)
#pragma unroll
                        for (int c = 0; c < 4; ++c) w[c] = fp8_pack_finite(piece(mi, 0, g, c), inv);
                    else
#pragma unroll
                        for (int c = 0; c < 4; ++c) w[c] = fp8_pack(piece(mi, 0, g, c), inv);
                    const int col = column(g);
                    if (col < N) {
                        u32x4* const to = reinterpret_cast<u32x4*>(static_cast<uint8_t*>(P.y) + (int64_t)m * N + col);
                        if (past) __builtin_nontemporal_store(w, to);
                        else *to = w;
                    }
                }
            }
        }
    }
}

template <int MODE, int BM, int BN, int WGM, int WGN, int KS, int STAGES, bool GATED, bool OUT8, bool GUARD>
__global__ __launch_bounds__(64 * WGM * WGN * KS, (cols_lds_chunks<MODE != COLS_BF16, BM, BN, WGN, STAGES, OUT8>() * 16 <= 80 * 1024 ? 2 : 1)) void cols_kernel(const ColsProblem P) {
    __shared__ u32x4 lds[cols_lds_chunks<MODE != COLS_BF16, BM, BN, WGN, STAGES, OUT8>()];
    const int total = P.tiles_m * P.tiles_n, per = (total + 7) >> 3;
    const int tile = (int)(blockIdx.x & 7) * per + (int)(blockIdx.x >> 3);
    if (tile >= total) return;
    cols_tile<MODE, BM, BN, WGM, WGN, KS, STAGES, GATED, OUT8, GUARD>(P, tile, lds);
}

// Few rows (one token's, a guidance pair's, a short text's).  A workgroup has 16 MB rows and 16 NB columns (of a gated product of value and gate each); its eight wavefronts take every eighth
// step of 128 bytes and bring the rows of P and Q straight into the registers as MFMA operands, U steps at once, and meet in LDS when they are done.  Bound by Q, which comes in once per
// 16 MB rows, and by trips to HBM one after the other: one for every eight U steps, and those of the epilogue's operands (a bias is widened where it is loaded, which waits for the steps before it; then the gate's, or
// the residual, is asked for).
constexpr int FEW_NW = 8;
template <bool FP8, bool GATED, int MB, int NB, int U>
__global__ __launch_bounds__(64 * FEW_NW) void few_rows_kernel(const ColsProblem P) {
    constexpr int NW = FEW_NW, QB = GATED ? 2 * NB : NB, BLOCKS = MB * QB, OUT = MB * NB, PER = (OUT + NW - 1) / NW;
    __shared__ f32x4 sh[NW * BLOCKS * 64];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int l16 = lane & 15, quad = lane >> 4;
    const int M = P.M, N = P.N, Kb = P.Kb;
    const int n0 = blockIdx.x * (16 * NB), m0 = blockIdx.y * (16 * MB);
    const uint8_t *qr[QB], *pr[MB], *qsr[QB], *psr[MB];
    f32x4 acc[MB][QB];
#pragma unroll
    for (int n = 0; n < QB; ++n) {
        const int64_t r = min(n0 + n % NB * 16 + l16, N - 1) + (n >= NB ? (int64_t)N : 0);
        qr[n] = P.q + r * Kb + quad * 16;
        if (FP8) qsr[n] = P.qs + r;
    }
#pragma unroll
    for (int m = 0; m < MB; ++m) {
        const int64_t r = min(m0 + m * 16 + l16, M - 1);
        pr[m] = P.p + r * Kb + quad * 16;
        if (FP8) psr[m] = P.ps + r;
#pragma unroll
        for (int n = 0; n < QB; ++n) acc[m][n] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
    const int steps = (Kb + 127) / 128;
    const u32x4 none = {0u, 0u, 0u, 0u};
    u32x4 qf[U][QB][2], pf[U][MB][2];
    uint32_t qsc[U][QB], psc[U][MB];
    auto fetch = [&](int s0) {
#pragma unroll
        for (int i = 0; i < U; ++i) {
            const int s = s0 + i * NW, k = s * 128;
            const bool lo = k + quad * 16 < Kb, hi = k + quad * 16 + 64 < Kb;      // (a chunk of 16 bytes is whole or not there)
#pragma unroll
            for (int n = 0; n < QB; ++n) {
                qf[i][n][0] = lo ? *reinterpret_cast<const u32x4*>(qr[n] + k) : none;
                qf[i][n][1] = hi ? *reinterpret_cast<const u32x4*>(qr[n] + k + 64) : none;
                if (FP8) qsc[i][n] = s < steps ? qsr[n][s * P.ldqs] : 127u;
            }
#pragma unroll
            for (int m = 0; m < MB; ++m) {
                pf[i][m][0] = lo ? *reinterpret_cast<const u32x4*>(pr[m] + k) : none;
                pf[i][m][1] = hi ? *reinterpret_cast<const u32x4*>(pr[m] + k + 64) : none;
                if (FP8) psc[i][m] = s < steps ? psr[m][s * P.ldps] : 127u;
            }
        }
    };
    fetch(wave);
    // what the epilogue adds, behind the first loads: wavefront w finishes blocks w, w + 8, ..., a lane has four columns of one row
    f32x4 bv[PER], bg[GATED ? PER : 1], rv[PER];
    auto place = [&](int i, int& row, int& col) {
        const int b = wave + i * NW;
        row = m0 + b / NB * 16 + l16;
        col = n0 + b % NB * 16 + quad * 4;
        return b < OUT && row < M && col < N;
    };
    auto read4 = [&](auto* p, int col) {
        if (col + 4 <= N) return load4(p);
        f32x4 v = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int e = 0; e < 3; ++e)
            if (col + e < N) v[e] = (float)p[e];
        return v;
    };
    auto write4 = [&](auto* p, int col, f32x4 v) {
        using T = std::remove_pointer_t<decltype(p)>;
        if (col + 4 <= N) store4(p, v);
        else
#pragma unroll
            for (int e = 0; e < 3; ++e)
                if (col + e < N) p[e] = (T)v[e];
    };
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        bv[i] = rv[i] = f32x4{0.f, 0.f, 0.f, 0.f};
        if (GATED) bg[GATED ? i : 0] = bv[i];
        int row, col;
        if (!place(i, row, col)) continue;
        const int64_t at = (int64_t)row * N + col;
        const __bf16* const bb = reinterpret_cast<const __bf16*>(P.bias) + col;
        if (P.bias) {
            bv[i] = read4(bb, col);
            if (GATED) bg[GATED ? i : 0] = read4(bb + N, col);
        }
        if (!GATED && P.res) rv[i] = P.y_f32 ? read4(static_cast<const float*>(P.res) + at, col) : read4(static_cast<const __bf16*>(P.res) + at, col);
    }
    for (int s0 = wave;;) {
#pragma unroll
        for (int i = 0; i < U; ++i) {
            if constexpr (FP8) {
                bf16x8 qw[QB][4];
#pragma unroll
                for (int n = 0; n < QB; ++n) widen32(qf[i][n], qsc[i][n], qw[n]);
#pragma unroll
                for (int m = 0; m < MB; ++m) {
                    bf16x8 pw[4];
                    widen32(pf[i][m], psc[i][m], pw);
#pragma unroll
                    for (int n = 0; n < QB; ++n)
#pragma unroll
                        for (int h = 0; h < 4; ++h) acc[m][n] = mfma_bf16(qw[n][h], pw[h], acc[m][n]);
                }
            } else {
#pragma unroll
                for (int m = 0; m < MB; ++m)
#pragma unroll
                    for (int n = 0; n < QB; ++n)
#pragma unroll
                        for (int h = 0; h < 2; ++h) acc[m][n] = mfma_bf16(__builtin_bit_cast(bf16x8, qf[i][n][h]), __builtin_bit_cast(bf16x8, pf[i][m][h]), acc[m][n]);
            }
        }
        s0 += NW * U;
        if (s0 >= steps) break;
        fetch(s0);
    }
#pragma unroll
    for (int b = 0; b < BLOCKS; ++b) sh[(wave * BLOCKS + b) * 64 + lane] = acc[b / QB][b % QB];
    __syncthreads();
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        int row, col;
        if (!place(i, row, col)) continue;
        const int b = (wave + i * NW) / NB * QB + (wave + i * NW) % NB;
        auto total = [&](int blk) {
            f32x4 v = sh[blk * 64 + lane];
#pragma unroll
            for (int w = 1; w < NW; ++w) v += sh[(w * BLOCKS + blk) * 64 + lane];
            return v;
        };
        f32x4 v[1] = {total(b) + bv[i]};
        const int64_t at = (int64_t)row * N + col;
        if constexpr (GATED) {
            f32x4 g[1] = {total(b + NB) + bg[i]};
            if (P.z) {
                __bf16* const zp = reinterpret_cast<__bf16*>(P.z) + (int64_t)row * 2 * N + col;
                write4(zp, col, v[0]);
                write4(zp + N, col, g[0]);
            }
            apply_act(P.act, g);
            v[0] *= g[0];
        } else {
            apply_act(P.act, v);
            v[0] += rv[i];
        }
        if (P.y_f32) write4(static_cast<float*>(P.y) + at, col, v[0]);
        else write4(static_cast<__bf16*>(P.y) + at, col, v[0]);
    }
}

// ---- launches
// (threads of a launch stay below 2^32)
inline bool cols_too_many(int64_t M, int64_t N, bool gated) { return ((M + 63) / 64) * (((gated ? 2 : 1) * N + 63) / 64) >= 1 << 22; }

// Which tiles: the ones whose launch is taken to be the shortest, us.  `slots` workgroups fit the chip; every full round of them takes rest + step for each 128 bytes of K, and so does
// the last, or, with no more than a workgroup a CU where there is room for two, alone_rest and alone_step.  (Fitted to launches of 16 to 8192 rows and five widths and depths from 320 to 5120 each, cold: off by
// 6 to 17 %, but what matters is which is least.)
struct ColsTile { int bm, bn, slots; float base, rest, step, alone_rest, alone_step; };
template <int TILES>
inline int cols_choose(const ColsTile (&tiles)[TILES], int64_t M, int64_t columns, int64_t Kb, float& least) {
    int best = 0;
    least = 0.f;
    const float steps = (float)((Kb + 127) / 128);
    for (int i = 0; i < TILES; ++i) {
        const ColsTile& t = tiles[i];
        const int64_t n = ((M + t.bm - 1) / t.bm) * ((columns + t.bn - 1) / t.bn), left = n % t.slots;
        const float us = t.base + (float)(n / t.slots + (left > 256 ? 1 : 0)) * (t.rest + steps * t.step) + (left > 0 && left <= 256 ? t.alone_rest + steps * t.alone_step : 0.f);
        if (i == 0 || us < least) best = i, least = us;
    }
    return best;
}
template <int MODE, int BM, int BN, int WGM, int WGN, int STAGES, bool GATED, bool OUT8, int KS = 1>
static int launch_cols(ColsProblem& P, hipStream_t stream) {
    constexpr int BN_OUT = GATED ? BN / 2 : BN;
    P.tiles_m = (P.M + BM - 1) / BM;
    P.tiles_n = (P.N + BN_OUT - 1) / BN_OUT;
    const int64_t tiles = (int64_t)P.tiles_m * P.tiles_n;
    const bool guard = P.Kb % 128 != 0;
    if (SD_DRY_RUN("gemm cols%s%s%s %dx%d/%d waves/%d stages%s; ", MODE == COLS_BF16 ? "" : MODE == COLS_FP8 ? " 8 bits" : " 8 bits wide", GATED ? " gated" : "", OUT8 ? " to 8 bits" : "", BM, BN, WGM * WGN * KS, STAGES, guard ? " guard" : "")) return SD_OK;
    const dim3 grid((unsigned)((tiles + 7) & ~7ll)), block(64 * WGM * WGN * KS);
    if (guard) hipLaunchKernelGGL((cols_kernel<MODE, BM, BN, WGM, WGN, KS, STAGES, GATED, OUT8, true>), grid, block, 0, stream, P);
    else hipLaunchKernelGGL((cols_kernel<MODE, BM, BN, WGM, WGN, KS, STAGES, GATED, OUT8, false>), grid, block, 0, stream, P);
    SD_HIP_CHECK(hipGetLastError());
    return SD_OK;
}
template <bool FP8, bool GATED, int MB, int NB, int U>
static int launch_few(const ColsProblem& P, hipStream_t stream) {
    if (SD_DRY_RUN("few rows%s%s %dx%d; ", FP8 ? " 8 bits" : "", GATED ? " gated" : "", 16 * MB, 16 * NB)) return SD_OK;
    hipLaunchKernelGGL((few_rows_kernel<FP8, GATED, MB, NB, U>), dim3((P.N + 16 * NB - 1) / (16 * NB), (P.M + 16 * MB - 1) / (16 * MB)), dim3(64 * FEW_NW), 0, stream, P);
    SD_HIP_CHECK(hipGetLastError());
    return SD_OK;
}

}  // namespace sd
