// Grouped bf16 MFMA GEMM for gfx950 with the rank-r LoRA update fused into the main loop.
//
// Every projection of the transformer block is y = x W^T (+ bias) with an optional LoRA
// term scale * (x A^T) B^T (Section 2, "Low-Rank Adaptation").  The down-projection
// t = scale * x A^T is a small GEMM of its own; the up-projection then rides in the base
// GEMM's K loop: [x | t] [W | B]^T, i.e. a second K segment of length r.  Both run in one
// launch: the down-projection's tiles come first in the grid and raise a flag per row block,
// and a base-GEMM tile looks at its flag only when it reaches the second K segment.
// Epilogues: bias, exact-erf GEGLU (Section 4.3's fused GEGLU), residual add, bf16 or fp32
// store.
//
// Tiling: BM x BN output tile per workgroup, BK = 64, WGM x WGN wavefronts, each owning
// (BM/WGM) x (BN/WGN) as 16x16x32 bf16 MFMA tiles with fp32 accumulators (32x32x16 ones cost more
// energy, and the chip lowers its clock under them: 8192x4096x4096 223 -> 211 us, 16384x1280x5120 + 64 249 -> 240, 8 x 4096 rows of
// 640 channels with four adapters 43.4 -> 42.6, 5000x640x2560 + 64 28.4 -> 26.8; same bits.  Some of the launches with one tile per CU are slower, and why is not known:
// 3000x1280x5120 + 64 55.5 -> 57.7, 6000x640x1280 + 64 21.0 -> 21.6, 4120x640x320 + 64 10.7 -> 10.9).
// Pipeline: operand tiles go global -> LDS directly (wave-wide 1 KB loads of 16-byte
// chunks, XOR-swizzled so the 16 rows one MFMA operand read touches fall in distinct
// banks) into a ring of STAGES tiles, STAGES-1 of them in flight ahead of the one being
// multiplied; operand blocks are read from LDS a few MFMAs ahead of their use,
// across the edge of two tiles too, and a tile's loads are dealt between the MFMAs of a
// step.  What bounds it: the L2 -> LDS operand stream, 100-125 GB/s per CU with all of them at it
// (a stream alone: 145 with few CUs), then the MFMAs, whose rate under load is 1.6 PFLOP/s; the
// two overlap only as far as no wavefront waits to issue a load.  8192x4096x4096, 128x128 tiles,
// eight wavefronts, three loads a burst after each barrier 271 us, dealt 248; 2048x1280x5120 + 64
// at one 128x128 tile per CU 51 and 41.  The epilogue stages 32-row x 64-column pieces of a wave's
// accumulators through LDS so that global stores (and residual loads) are 16-byte rows.
#pragma once
#include "gemm_dma.hpp"

namespace sd {

constexpr int EPI_STRIDE = 68;   // floats per staged row: 16 rows apart by 4 banks, 16 bytes of each

// Tiles that gave up waiting for a producer's flag (never, unless the dependency protocol is
// broken): the wait is bounded so that every wavefront exits whatever happens.
static __device__ unsigned long long g_gemm_dep_timeouts = 0;   // (the projections' launches, gemm.hip)
constexpr int DEP_SPIN_LIMIT = 1 << 19;
struct DeviceMem {
    __device__ __forceinline__ static uint64_t load64(const uint64_t* p) { return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }
    __device__ __forceinline__ static void store64(uint64_t* p, uint64_t v) { __hip_atomic_store(p, v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }
    __device__ __forceinline__ static void store32(int32_t* p, int32_t v) { __hip_atomic_store(p, v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }
    __device__ __forceinline__ static int32_t add32(int32_t* p, int32_t v) { return __hip_atomic_fetch_add(p, v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }
};
// Tiles of signalling problems (down-projections, N = rank) run a body of their own inside the
// same kernel: BN = 64 instead of the launch's BN, which frees LDS for a deeper ring.  Other
// tiles of the launch wait for these, and what a down-projection tile spends is latency per
// k-step, so tiles in flight are what shortens it.
constexpr int DOWN_BN = 64;
template <int BM, int BN, int BK, int STAGES>
constexpr int down_stages() {
    if (BN <= DOWN_BN) return STAGES;
    const int fit = STAGES * (BM + BN) / (BM + DOWN_BN);   // stages of the narrower tile in the same bytes
    return fit > 5 ? 5 : (fit < 3 ? 3 : fit);
}
template <int BM, int BN, int BK, int WGM, int WGN, int STAGES>
constexpr int gemm_lds_chunks() {
    constexpr int ring = STAGES * (BM + BN) * (BK / 8);
    constexpr int dring = down_stages<BM, BN, BK, STAGES>() * (BM + (BN < DOWN_BN ? BN : DOWN_BN)) * (BK / 8);
    constexpr int epi = WGM * WGN * 32 * EPI_STRIDE / 4;
    constexpr int m = ring > dring ? ring : dring;
    return m > epi ? m : epi;
}

// What a launch does beyond a projection of the block.
//   act: a linear layer's, y = act(z) + residual, z the product with its bias, and z itself kept in bf16, laid out as y, where asked for.
//   pt, qt: an operand whose rows are the reduction's, p0 [K0, Mp] or q0 [K0, N] (the two products of a backward pass).  Its
//   stages are BK rows of BM or BN elements in LDS, and the transposing LDS read hands a lane the elements of one
//   column.  One segment, and rows of the operand that are a multiple of 8 elements long.
struct GemmPlain { static constexpr bool act = false, pt = false, qt = false; };
template <bool PT, bool QT>
struct GemmTransposed { static constexpr bool act = false, pt = PT, qt = QT; };
struct GemmAct { static constexpr bool act = true, pt = false, qt = false; };
// Which 32-byte piece of an LDS row of W elements holds logical piece u of row k: u ^ tr_swz<W>(k).  The four rows that 16 lanes
// read a piece of each, and those eight rows further that the next 16 do, lie in distinct banks.
template <int W>
__device__ __forceinline__ int tr_swz(int k) {
    return W == 64 ? (((k >> 1) & 1) << 1) | ((k >> 3) & 1) : (k & 3) | (((k >> 3) & 1) << 2);
}

// GUARD: K segments that are not multiples of 64 (tail chunks read zeros).
// Two workgroups per CU whenever the ring leaves room for it (LDS <= 80 KB): the register
// budget is then 256 per lane (accumulators in AGPRs, the rest in VGPRs).
template <int BM, int BN, int BK, int WGM, int WGN, int STAGES>
constexpr int gemm_min_waves() {
    return gemm_lds_chunks<BM, BN, BK, WGM, WGN, STAGES>() * 16 <= 80 * 1024 ? 2 : 1;
}

// 16-column blocks of a wavefront that the epilogue stages and stores at a time, of `nout` that it has
constexpr int gemm_pass_blocks(int nout) { return nout % 4 == 0 ? 4 : nout % 2 == 0 ? 2 : 1; }
// A linear layer's large z goes past the caches, which y, that the next call reads, then has to itself: z waits for the backward pass.  (us, the layers of a feed-forward, layer norm and both products,
// 8192 x 1280 to 5120 287 / 278, 6144 198 / 193, 16384 x 640 to 2560 180 / 175; but 4096 x 1280 to 5120 156 / 174, where the caches hold z too.)  Passes of 64 columns write whole lines
// of it; those of 16, which the 128x160 tiles' wavefronts have, do not, and then the caches have to join them (past / through them: 42496x960x320 131 / 82, 88576x320x1280 149 / 125).
template <int NOUT>
__host__ __device__ constexpr bool gemm_z_past(int64_t rows, int64_t ldy) { return gemm_pass_blocks(NOUT) == 4 && rows * ldy > (24ll << 20); }

template <int BM, int BN, int BK, int WGM, int WGN, int STAGES, bool GEGLU, bool GUARD, bool RES32, class Ext>
__device__ __forceinline__ void gemm_tile(const GemmProblem& P, const int tile, u32x4* const lds, const Ext) {
    constexpr int NW = WGM * WGN;
    constexpr int WM = BM / WGM, WN = BN / WGN;
    constexpr int MI = WM / 16, NI = WN / 16;  // 16x16 blocks of a wavefront
    constexpr int CPR = BK / 8;                // 16-byte chunks per LDS row
    constexpr int RPB = 64 / CPR;              // tile rows per 1 KB block (one wave-wide load)
    constexpr int SLOTS = 2 * NI;              // a tile is two 32 deep k-steps of NI blocks of Q; a slot multiplies one of them by the MI blocks of P
    constexpr int RING = NI < 4 || NI % 2 ? NI : 4;   // blocks of Q in registers
    constexpr int NBLK = (BM + BN) / RPB;      // 1 KB blocks per stage
    constexpr int LPT = NBLK / NW;             // direct-to-LDS loads per wave (= per lane) per tile
    constexpr int STAGE = (BM + BN) * CPR;     // 16-byte chunks per stage
    static_assert(BK == 64 && SLOTS % RING == 0, "BK");
    static_assert(NBLK % NW == 0, "tile/waves mismatch");
    static_assert(!GEGLU || (NI % 2 == 0), "GEGLU needs value/gate column-block pairs per wave");
    static_assert(STAGES >= 2 && STAGES <= 5, "ring depth");

    // ---- which tile of the problem ----
    const int local = tile - P.tile_begin;
    const int band_tiles = 8 * P.tiles_n;
    const int band = local / band_tiles, rem = local - band * band_tiles;
    const int band_rows = min(8, P.tiles_m - band * 8);
    const int tn = rem / band_rows, tm = band * 8 + rem % band_rows;
    constexpr int BN_OUT = GEGLU ? BN / 2 : BN;
    const int m0 = tm * BM, n0 = tn * BN_OUT;
    const int Mp = P.Mp, N = P.N, K0 = P.K0, K1 = P.K1;
    const int nk0 = (K0 + BK - 1) / BK, nk1 = (K1 + BK - 1) / BK, nkt = nk0 + nk1;

    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int l16 = lane & 15, quad = lane >> 4;
    const int wm = (wave / WGN) * WM, wn = (wave % WGN) * WN;

    // ---- dependency on a producer problem of this launch.  The flags are read once now (the
    // answer arrives with the first operand tile); tiles that start after the producer has
    // finished, the usual case, never look again.  Device-scope loads: the producer's tile may
    // have run on another XCD.
    const int32_t* const wflag = std::is_same_v<Ext, GemmPlain> && K1 ? P.wait : nullptr;
    const int32_t* fptr = nullptr;
    // with a nonce: the record of this row block, and the word of it that this lane looks at
    uint64_t* const rec = wflag && P.nonce ? reinterpret_cast<uint64_t*>(const_cast<int32_t*>(wflag)) + tm * (DEP_RECORD / 8) : nullptr;
    const uint64_t* const rword = rec + dep_record_word(lane, P.wait_need);
    bool f_early = true;
    if (rec) {
        f_early = dep_record_ready(lane, P.wait_need, DeviceMem::load64(rword), P.nonce);
    } else if (wflag) {
        const int lo = P.wait_cols ? n0 : m0;
        const int hi = P.wait_cols ? min(n0 + BN_OUT, N) : min(m0 + BM, Mp);
        const int f0 = lo / BM, f1 = (hi - 1) / BM;
        fptr = wflag + f0 + min(lane, f1 - f0);
        f_early = __hip_atomic_load(fptr, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) >= P.wait_need;
    }

    // Q-operand (weight) row of tile row j.  GEGLU: 16-row blocks alternate value / gate
    // rows of the same 16 output columns, so one lane ends up holding both halves.
    auto qrow = [&](int j) -> int {
        if (GEGLU) {
            int blk = j >> 4;
            int col = n0 + (blk >> 1) * 16 + (j & 15);
            col = col < N ? col : N - 1;
            return col + ((blk & 1) ? P.geglu_F : 0);
        } else {
            int col = n0 + j;
            return col < N ? col : N - 1;
        }
    };

    // ---- loader.  Load j of wave w fills 1 KB block (j*NW + w) of a stage: RPB tile rows
    // (P rows first, then Q rows) of CPR chunks; lane l lands at chunk position l % CPR of row
    // l / CPR, so it must fetch the logical chunk that the XOR swizzle places there.  The
    // first JP loads of a lane are P rows, the rest Q rows; a lane's source is a wave-uniform
    // base (operand start + k offset of the step, scalar arithmetic) plus a constant 32-bit
    // byte offset (row, chunk).
    constexpr int JP = (BM / RPB) / NW;
    static_assert((BM / RPB) % NW == 0, "P/Q split must fall on a load index");
    uint32_t off0[LPT];          // byte offset of this lane's chunk from the operand start, K segment 0
    uint32_t off1[LPT];          // ... K segment 1 (LoRA); equals off0 when there is none
    int kcol[GUARD ? LPT : 1];   // first k of that chunk within a tile (only partial tiles need it)
    const uint16_t* const pb0 = P.p0 + (Ext::pt ? (int64_t)m0 : (int64_t)m0 * P.ldp0);
    const uint16_t* const pb1 = K1 ? P.p1 + (int64_t)m0 * P.ldp1 : pb0;
    const uint16_t* const qb0 = P.q0 + (Ext::qt ? (int64_t)n0 : (int64_t)n0 * P.ldq0);
    // elements between an operand's k-steps of depth one
    const int64_t pstep = Ext::pt ? P.ldp0 : 1, qstep = Ext::qt ? P.ldq0 : 1;
    const uint16_t* const qb1 = K1 ? P.q1 + (int64_t)n0 * P.ldq1 : qb0;
    {
        const int64_t ldp0 = P.ldp0, ldq0 = P.ldq0;
        const int64_t ldp1 = K1 ? P.ldp1 : P.ldp0, ldq1 = K1 ? P.ldq1 : P.ldq0;
#pragma unroll
        for (int j = 0; j < LPT; ++j) {
            const int row = (j * NW + wave) * RPB + lane / CPR;    // row within the stage
            const int c = swz<CPR>(row, lane % CPR);               // logical chunk fetched by this lane
            if (GUARD) kcol[j] = c * 8;
            if ((j < JP && Ext::pt) || (j >= JP && Ext::qt)) {
                constexpr int WP = Ext::pt ? BM : 64, WQ = Ext::qt ? BN : 64;   // elements of an LDS row
                const int w = j < JP ? WP : WQ, blk = j < JP ? j * NW + wave : j * NW + wave - BM / RPB;
                const int k = blk * (512 / w) + lane / (w / 8), pos = lane % (w / 8);
                const int piece = (pos >> 1) ^ (j < JP ? tr_swz<WP>(k) : tr_swz<WQ>(k));
                // (columns past the end: the last eight that there are)
                const int first = j < JP ? m0 : n0, last = ((j < JP ? Mp : N) - 1) & ~7;
                const int col = min(first + piece * 16 + (pos & 1) * 8, last) - first;
                off0[j] = off1[j] = (uint32_t)((k * (j < JP ? ldp0 : ldq0) + col) * 2);
                if (GUARD) kcol[j] = k;
            } else if (j < JP) {
                int r = m0 + row;
                r = (r < Mp ? r : Mp - 1) - m0;
                off0[j] = (uint32_t)((r * ldp0 + c * 8) * 2);
                off1[j] = (uint32_t)((r * ldp1 + c * 8) * 2);
            } else {
                const int qr = qrow(row - BM) - n0;
                off0[j] = (uint32_t)((qr * ldq0 + c * 8) * 2);
                off1[j] = (uint32_t)((qr * ldq1 + c * 8) * 2);
            }
        }
    }
    const uint32_t lds_base = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) void*)lds;
    const uint32_t wave_base = lds_base + (uint32_t)wave * 1024;
    // issue the loads of k-step t into ring stage `stg`.  A partial last tile of a segment
    // (GUARD only) takes per-lane 64-bit addresses so that chunks past the segment's end can
    // point at the zero page.
    bool dep_ready = wflag == nullptr;
    bool timed_out = false;      // this wavefront gave up waiting: its output is poisoned below
    auto issue_tile = [&](int t, int stg) {
        const bool s1 = t >= nk0;
        const int kb = (s1 ? t - nk0 : t) * BK;
        const int Kseg = s1 ? K1 : K0;
        const uint32_t sbase = wave_base + (uint32_t)stg * (STAGE * 16);
        const uint16_t* pb = (s1 ? pb1 : pb0) + (Ext::pt ? kb * pstep : (int64_t)kb);
        const uint16_t* qb = (s1 ? qb1 : qb0) + (Ext::qt ? kb * qstep : (int64_t)kb);
        const bool dev = s1 && wflag;   // segment 1 was written during this launch
        if (dev && !dep_ready) {
            // the producer's tiles were dispatched before this one and wait for nothing, so
            // this ends; the bound is there so that it ends even if that reasoning is wrong
            for (int spins = 0;; ++spins) {
                bool seen, given_up = false;
                if (rec) {
                    const uint64_t v = DeviceMem::load64(rword);
                    seen = dep_record_ready(lane, P.wait_need, v, P.nonce);
                    given_up = dep_record_given_up(lane, P.wait_need, v, P.nonce);
                } else {
                    seen = __hip_atomic_load(fptr, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) >= P.wait_need;
                }
                if (__all(seen)) break;
                if (spins >= DEP_SPIN_LIMIT || __any(given_up)) {
                    if (tid == 0) atomicAdd(&g_gemm_dep_timeouts, 1ull);
                    if (rec && lane == 0) DepRecord<DeviceMem>::give_up(rec, P.nonce);
                    timed_out = true;
                    break;
                }
                __builtin_amdgcn_s_sleep(8);
            }
            dep_ready = true;
        }
        if (GUARD && kb + BK > Kseg) {
#pragma unroll
            for (int j = 0; j < LPT; ++j) {
                const char* src = reinterpret_cast<const char*>(j < JP ? pb : qb) + (s1 ? off1[j] : off0[j]);
                src = (kb + kcol[GUARD ? j : 0] < Kseg) ? src : reinterpret_cast<const char*>(g_gemm_zeros);
                if (dev) dma16<true>(src, sbase + (uint32_t)j * (NW * 1024));
                else dma16<false>(src, sbase + (uint32_t)j * (NW * 1024));
            }
        } else if (dev) {
#pragma unroll
            for (int j = 0; j < LPT; ++j)
                dma16_so<true>(j < JP ? pb : qb, off1[j], sbase + (uint32_t)j * (NW * 1024));
        } else {
#pragma unroll
            for (int j = 0; j < LPT; ++j)
                dma16_so<false>(j < JP ? pb : qb, s1 ? off1[j] : off0[j], sbase + (uint32_t)j * (NW * 1024));
        }
    };

    f32x4 acc[MI][NI];
#pragma unroll
    for (int mi = 0; mi < MI; ++mi)
#pragma unroll
        for (int ni = 0; ni < NI; ++ni) acc[mi][ni] = f32x4{0.f, 0.f, 0.f, 0.f};

    // operands in registers: the P blocks of both k-steps, and a ring of Q blocks.  Slot s multiplies Q block s % NI in k-step
    // s / NI out of bfr[s % RING], which is then refilled for slot s + RING, over the edge between two tiles too.
    // The MFMA takes the Q rows first: a lane holds four consecutive columns of one row of the result.
    bf16x8 af[2][MI], bfr[RING];
    const int lrow = l16 * CPR, lsw = (l16 >> 1) & 7;       // (rows 16 apart share the swizzle)
    auto frag = [&](int st, int ks) { return lds + (st * STAGE + lrow + ((ks * 4 + quad) ^ lsw)); };
    // Transposed operands: 16 lanes read 32 bytes of each of four rows, and each gets one column of them; twice for the eight k of
    // a lane.  Rows 8 quad + 4 h + l16 / 4 of a k-step share their swizzle.
    typedef __attribute__((address_space(3))) char lds_char;
    lds_char* const lds8 = (lds_char*)lds;
    auto tr_row = [&](int w) { return (quad * 8 + (l16 >> 2)) * w * 2 + ((l16 >> 1) & 1) * 16 + (l16 & 1) * 8; };
    auto tr_read = [&](int at, int w) {
        const bf16x4 a = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((__attribute__((address_space(3))) bf16x4*)(lds8 + at));
        const bf16x4 b = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((__attribute__((address_space(3))) bf16x4*)(lds8 + at + 4 * w * 2));
        return __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7);
    };
    int tp[Ext::pt ? MI : 1], tq[Ext::qt ? NI : 1];         // where in a k-step of a stage a lane's piece of each block is
    if constexpr (Ext::pt)
#pragma unroll
        for (int mi = 0; mi < MI; ++mi) tp[mi] = tr_row(BM) + (((wm / 16 + mi) ^ tr_swz<BM>(quad * 8 + (l16 >> 2))) << 5);
    if constexpr (Ext::qt)
#pragma unroll
        for (int ni = 0; ni < NI; ++ni) tq[ni] = BM * BK * 2 + tr_row(BN) + (((wn / 16 + ni) ^ tr_swz<BN>(quad * 8 + (l16 >> 2))) << 5);
    auto fetch_p = [&](int st, int ks) {
        if constexpr (Ext::pt) {
#pragma unroll
            for (int mi = 0; mi < MI; ++mi) af[ks][mi] = tr_read(tp[mi] + st * (STAGE * 16) + ks * 32 * BM * 2, BM);
        } else {
            const u32x4* const la = frag(st, ks) + wm * CPR;
#pragma unroll
            for (int mi = 0; mi < MI; ++mi) af[ks][mi] = __builtin_bit_cast(bf16x8, la[mi * 16 * CPR]);
        }
    };
    auto fetch_q = [&](int st, int s) {
        if constexpr (Ext::qt) bfr[s % RING] = tr_read(tq[s % NI] + st * (STAGE * 16) + s / NI * 32 * BN * 2, BN);
        else bfr[s % RING] = __builtin_bit_cast(bf16x8, (frag(st, s / NI) + (BM + wn) * CPR)[(s % NI) * 16 * CPR]);
    };
    auto multiply = [&](int s) {
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int mi = 0; mi < MI; ++mi)
            acc[mi][s % NI] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(bfr[s % RING], af[s / NI][mi], acc[mi][s % NI], 0, 0, 0);
        __builtin_amdgcn_sched_barrier(0);
    };
    // A step: the last RING slots of a tile, whose operands are in registers, while the first of the next (in stage sn) are read
    // (`edge`); then the others of that one (`head`).  The loads of another tile are dealt over it, a few behind each
    // slot's MFMAs (`load(j)` issues one): a wavefront issues in order, and a burst of loads would hold up its
    // MFMAs until the address unit has taken the last one, at 16 clocks apiece for the whole CU.
    auto deal = [&](auto load, int i) {
#pragma unroll
        for (int j = i * LPT / SLOTS; j < (i + 1) * LPT / SLOTS; ++j) load(j);
    };
    auto edge = [&](int sn, auto load) {
        fetch_p(sn, 0);
#pragma unroll
        for (int i = 0; i < RING; ++i) {
            multiply(SLOTS - RING + i);
            deal(load, i);
            fetch_q(sn, i);
        }
    };
    auto head = [&](int st, auto load) {
#pragma unroll
        for (int s = 0; s < SLOTS - RING; ++s) {
            if (s == 0) fetch_p(st, 1);
            multiply(s);
            deal(load, RING + s);
            fetch_q(st, s + RING);
        }
    };
    auto no_load = [](int) {};

    // ---- prologue: the first STAGES tiles in flight, the first fragments of tile 0 read
#pragma unroll
    for (int d = 0; d < STAGES; ++d)
        if (d < nkt) issue_tile(d, d);
    if (!dep_ready) dep_ready = __all(f_early);
    auto wait_tiles = [&](int newer) {   // `newer` tiles (at most STAGES - 1) may stay in flight
        if (STAGES >= 5 && newer >= 4) wait_vmcnt<4 * LPT>();
        else if (STAGES >= 4 && newer >= 3) wait_vmcnt<3 * LPT>();
        else if (STAGES >= 3 && newer >= 2) wait_vmcnt<2 * LPT>();
        else if (newer >= 1) wait_vmcnt<LPT>();
        else wait_vmcnt<0>();
    };
    wait_tiles(nkt - 1 < STAGES - 1 ? nkt - 1 : STAGES - 1);
    __syncthreads();
    fetch_p(0, 0);
#pragma unroll
    for (int s = 0; s < RING; ++s) fetch_q(0, s);
    head(0, no_load);

    // ---- main loop.  A step starts at the edge between tile t and tile t+1, before the MFMAs of
    // tile t's last slots: their operands are in registers, so once this wave's loads of tile t+1
    // have landed (newer ones may stay in flight) one barrier says both that tile t+1 is whole and
    // that the stage of tile t is free.  That stage is refilled with tile t+STAGES, its loads dealt
    // over the step.
    int st = 0;                         // stage of tile t
    int t = 0;
    const int nfull = GUARD ? K0 / BK : nk0;   // whole tiles of K segment 0
#pragma unroll 1
    for (; t + STAGES < nfull; ++t) {
        wait_vmcnt<(STAGES - 2) * LPT>();
        __syncthreads();
        const int sn = st + 1 == STAGES ? 0 : st + 1;
        const uint16_t* const pb = Ext::pt ? pb0 + (t + STAGES) * BK * pstep : pb0 + (t + STAGES) * BK;
        const uint16_t* const qb = Ext::qt ? qb0 + (t + STAGES) * BK * qstep : qb0 + (t + STAGES) * BK;
        const uint32_t sbase = wave_base + (uint32_t)st * (STAGE * 16);
        auto load = [&](int j) { dma16_so<false>(j < JP ? pb : qb, off0[j], sbase + (uint32_t)j * (NW * 1024)); };
        edge(sn, load);
        head(sn, load);
        st = sn;
    }
    // the same for the tiles around and behind the end of segment 0, and for the last ones, which
    // have nothing left to load and shrinking wait counts
#pragma unroll 1
    for (; t + 1 < nkt; ++t) {
        wait_tiles(nkt - 2 - t < STAGES - 2 ? nkt - 2 - t : STAGES - 2);
        __syncthreads();
        const int sn = st + 1 == STAGES ? 0 : st + 1;
        if (t + STAGES < nkt) issue_tile(t + STAGES, st);
        edge(sn, no_load);
        head(sn, no_load);
        st = sn;
    }

    // ---- epilogue geometry.  A lane holds columns 4*quad .. +4 of each of its 16-column blocks, in row l16 of each 16-row block.
    // Each wave stages a 32-row x CCOLS-column piece at a time in its own LDS region (fp32, padded rows) and writes it out as
    // whole row pieces: lane handles 4 consecutive columns (lcol) of row lr, lr + RPP, ... of the piece.  (Stored from where they are, 32 or 64 bytes
    // of a row at a time: 8192x1920x640 + 64 39 -> 44 us, 2048x1280x1280 + 64 with an fp32 residual 20.1 -> 21.9.)
    constexpr int NOUT = GEGLU ? NI / 2 : NI;   // 16-column output blocks per wave
    constexpr int CB = gemm_pass_blocks(NOUT);  // ... staged per pass (<= 64 columns)
    constexpr int CCOLS = CB * 16;              // staged columns
    constexpr int LPR = CCOLS / 4;              // lanes per staged row (4 columns each)
    constexpr int RPP = 64 / LPR;               // rows per pass
    constexpr int NPASS = 32 / RPP;
    static_assert(NOUT % CB == 0 && MI % 2 == 0, "pieces");
    const int wn_out = GEGLU ? (wn >> 1) : wn;
    const bool y_f32 = P.y_f32 != 0;
    const int lr = lane / LPR, lcol = (lane % LPR) * 4;
    const bool ld_ok = ((P.ldy & 3) == 0) && (!P.res || (P.ldr & 3) == 0);
    // a tile that lies inside the output with 16-byte-aligned rows takes straight-line code: all
    // staged pieces read, then all residual pieces, then all stores (no per-lane bounds)
    const bool full = ld_ok && m0 + BM <= Mp && n0 + BN_OUT <= N;
    const int qcol = n0 + wn_out + quad * 4;

    // fp32 residual: fetch this lane's pieces of the whole wave tile now, so that the loads
    // fly during the last tile's MFMAs and the epilogue never waits piece by piece
    f32x4 rpre[RES32 ? MI / 2 : 1][RES32 ? NOUT / CB : 1][RES32 ? NPASS : 1];
    const bool res_pre = RES32 && P.res && P.res_f32 && ld_ok;
    if (RES32 && res_pre) {
        const float* rp = static_cast<const float*>(P.res);
#pragma unroll
        for (int mi = 0; mi < MI / 2; ++mi)
#pragma unroll
            for (int cc = 0; cc < NOUT / CB; ++cc) {
                const int q4 = n0 + wn_out + cc * CCOLS + lcol;
#pragma unroll
                for (int pass = 0; pass < NPASS; ++pass) {
                    const int p = m0 + wm + mi * 32 + pass * RPP + lr;
                    f32x4 r = {0.f, 0.f, 0.f, 0.f};
                    if (p < Mp && q4 + 4 <= N) r = *reinterpret_cast<const f32x4*>(rp + (int64_t)p * P.ldr + q4);
                    rpre[RES32 ? mi : 0][RES32 ? cc : 0][RES32 ? pass : 0] = r;
                }
            }
    }
    // per-column bias of this lane's output columns: fetched now as well (raw bits, widened after
    // the last MFMAs; a column past N reads the last valid one and is never stored)
    const uint16_t* bias = P.bias;
    u32x2 bv_raw[NOUT], bg_raw[GEGLU ? NOUT : 1];
#pragma unroll
    for (int nj = 0; nj < NOUT; ++nj) {
        bv_raw[nj] = u32x2{0u, 0u};
        if (GEGLU) bg_raw[GEGLU ? nj : 0] = u32x2{0u, 0u};
    }
    if (bias && !P.bias_on_rows) {
        // (a record's bias need not be aligned; whole pieces of four where it is)
        const bool pieces = n0 + BN_OUT <= N && ((reinterpret_cast<uintptr_t>(bias) & 7) == 0) && (!GEGLU || (P.geglu_F & 3) == 0);
        auto four = [&](const uint16_t* b, int q4) {
            if (pieces) return *as_global(reinterpret_cast<const u32x2*>(b + q4));
            uint32_t w[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) w[e] = *as_global(b + min(q4 + e, N - 1));
            return u32x2{w[0] | (w[1] << 16), w[2] | (w[3] << 16)};
        };
#pragma unroll
        for (int nj = 0; nj < NOUT; ++nj) {
            bv_raw[nj] = four(bias, qcol + nj * 16);
            if (GEGLU) bg_raw[GEGLU ? nj : 0] = four(bias + P.geglu_F, qcol + nj * 16);
        }
    }
#pragma unroll
    for (int s = SLOTS - RING; s < SLOTS; ++s) multiply(s);
    __syncthreads();   // ring reads done before the epilogue reuses LDS
    // a record's last reader takes the nonce out again.  (Every wavefront of the tile has seen the words by
    // now, or has given up; the count was zeroed before the first of them was written.)
    int readers_before = -1;
    if (rec && tid == 0) readers_before = DepRecord<DeviceMem>::leave(rec);

    // ---- epilogue
    float* stage = reinterpret_cast<float*>(lds) + wave * 32 * EPI_STRIDE;
    // a wavefront that read its second K segment without the producer's flag stores NaN: what it
    // computed from a stale or half-written down-projection must not look like a result
    const float alpha = timed_out ? __builtin_nanf("") : P.alpha;
    const bool z_past = Ext::act && gemm_z_past<NOUT>(Mp, P.ldy);
    int32_t* const sig = std::is_same_v<Ext, GemmPlain> ? P.signal : nullptr;
    // (opaque to the optimiser, which would otherwise widen right after the loads and wait for them there)
#pragma unroll
    for (int nj = 0; nj < NOUT; ++nj) {
        asm volatile("" : "+v"(bv_raw[nj]));
        if (GEGLU) asm volatile("" : "+v"(bg_raw[GEGLU ? nj : 0]));
    }
    auto widen = [](const u32x2& w, int e) { return e & 1 ? bf16hi_to_f32(w[e >> 1]) : bf16lo_to_f32(w[e >> 1]); };
    // block (mi, nj) as it is staged
    auto value = [&](int mi, int nj) {
        f32x4 v;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            if (GEGLU) v[e] = (alpha * acc[mi][GEGLU ? 2 * nj : 0][e] + widen(bv_raw[nj], e)) * gelu_erf(alpha * acc[mi][GEGLU ? 2 * nj + 1 : 0][e] + widen(bg_raw[GEGLU ? nj : 0], e));
            else v[e] = alpha * acc[mi][nj][e] + widen(bv_raw[nj], e);
        }
        return v;
    };
#pragma unroll
    for (int mi = 0; mi < MI / 2; ++mi) {
#pragma unroll
        for (int cc = 0; cc < NOUT / CB; ++cc) {
            // 1) registers -> staging (value after alpha, bias, GEGLU)
#pragma unroll
            for (int m2 = 0; m2 < 2; ++m2)
#pragma unroll
                for (int cj = 0; cj < CB; ++cj)
                    *reinterpret_cast<f32x4*>(stage + (m2 * 16 + l16) * EPI_STRIDE + cj * 16 + quad * 4) = value(mi * 2 + m2, cc * CB + cj);
            __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
            __builtin_amdgcn_wave_barrier();
            // 2) staging -> global: lane handles 4 consecutive columns of one row per pass
            const int q4 = n0 + wn_out + cc * CCOLS + lcol;
            if (full) {
                f32x4 val[NPASS];
#pragma unroll
                for (int pass = 0; pass < NPASS; ++pass)
                    val[pass] = *reinterpret_cast<const f32x4*>(stage + (pass * RPP + lr) * EPI_STRIDE + lcol);
                const int p0 = m0 + wm + mi * 32 + lr;          // row of pass 0; pass k is RPP * k rows further
                if (bias && P.bias_on_rows) {
                    float br[NPASS];
#pragma unroll
                    for (int pass = 0; pass < NPASS; ++pass) br[pass] = bf16_to_f32(*as_global(bias + p0 + pass * RPP));
#pragma unroll
                    for (int pass = 0; pass < NPASS; ++pass) val[pass] += br[pass];
                }
                if constexpr (Ext::act) {
                    if (P.z) {
                        uint16_t* const zp = P.z + (int64_t)p0 * P.ldy + q4;
                        bf16x4 o[NPASS];
#pragma unroll
                        for (int pass = 0; pass < NPASS; ++pass)
#pragma unroll
                            for (int e = 0; e < 4; ++e) o[pass][e] = (__bf16)val[pass][e];
                        if (z_past) {
                            asm volatile("");       // (or the two kinds of store are merged into one)
#pragma unroll
                            for (int pass = 0; pass < NPASS; ++pass) __builtin_nontemporal_store(o[pass], as_global(reinterpret_cast<bf16x4*>(zp + (int64_t)(pass * RPP) * P.ldy)));
                            asm volatile("");
                        } else
#pragma unroll
                            for (int pass = 0; pass < NPASS; ++pass) *as_global(reinterpret_cast<bf16x4*>(zp + (int64_t)(pass * RPP) * P.ldy)) = o[pass];
                    }
                    apply_act(P.act(), val);
                }
                if (P.res) {
                    if (RES32 && res_pre) {
#pragma unroll
                        for (int pass = 0; pass < NPASS; ++pass) val[pass] += rpre[RES32 ? mi : 0][RES32 ? cc : 0][RES32 ? pass : 0];
                    } else if (P.res_f32) {
                        const float* rf = static_cast<const float*>(P.res) + (int64_t)p0 * P.ldr + q4;
                        f32x4 r[NPASS];
#pragma unroll
                        for (int pass = 0; pass < NPASS; ++pass) r[pass] = *as_global(reinterpret_cast<const f32x4*>(rf + (int64_t)(pass * RPP) * P.ldr));
#pragma unroll
                        for (int pass = 0; pass < NPASS; ++pass) val[pass] += r[pass];
                    } else {
                        const uint16_t* rb = static_cast<const uint16_t*>(P.res) + (int64_t)p0 * P.ldr + q4;
                        u32x2 r[NPASS];
#pragma unroll
                        for (int pass = 0; pass < NPASS; ++pass) r[pass] = *as_global(reinterpret_cast<const u32x2*>(rb + (int64_t)(pass * RPP) * P.ldr));
#pragma unroll
                        for (int pass = 0; pass < NPASS; ++pass) {
                            val[pass][0] += bf16lo_to_f32(r[pass][0]); val[pass][1] += bf16hi_to_f32(r[pass][0]);
                            val[pass][2] += bf16lo_to_f32(r[pass][1]); val[pass][3] += bf16hi_to_f32(r[pass][1]);
                        }
                    }
                }
                if (y_f32) {
                    float* yp = static_cast<float*>(P.y) + (int64_t)p0 * P.ldy + q4;
#pragma unroll
                    for (int pass = 0; pass < NPASS; ++pass) *as_global(reinterpret_cast<f32x4*>(yp + (int64_t)(pass * RPP) * P.ldy)) = val[pass];
                } else {
                    uint16_t* yp = static_cast<uint16_t*>(P.y) + (int64_t)p0 * P.ldy + q4;
#pragma unroll
                    for (int pass = 0; pass < NPASS; ++pass) {
                        bf16x4 o;
#pragma unroll
                        for (int e = 0; e < 4; ++e) o[e] = (__bf16)val[pass][e];
                        uint16_t* const yq = yp + (int64_t)(pass * RPP) * P.ldy;
                        if (sig)   // device-scope store: read by tiles of this launch on other XCDs
                            __hip_atomic_store(reinterpret_cast<uint64_t*>(yq), __builtin_bit_cast(uint64_t, o), __ATOMIC_RELAXED,
                                               __HIP_MEMORY_SCOPE_AGENT);
                        else
                            *as_global(reinterpret_cast<bf16x4*>(yq)) = o;
                    }
                }
            } else {
                const bool vec_ok = ld_ok && (q4 + 4 <= N);   // 16-byte path: whole piece inside N, aligned rows
#pragma unroll
                for (int pass = 0; pass < NPASS; ++pass) {
                    const int rr = pass * RPP + lr;
                    const int p = m0 + wm + mi * 32 + rr;
                    if (p < Mp && q4 < N) {
                        f32x4 val = *reinterpret_cast<const f32x4*>(stage + rr * EPI_STRIDE + lcol);
                        if (bias && P.bias_on_rows) val += bf16_to_f32(*as_global(bias + p));
                        if constexpr (Ext::act) {
                            if (P.z)
#pragma unroll
                                for (int e = 0; e < 4; ++e)
                                    if (q4 + e < N) *as_global(P.z + (int64_t)p * P.ldy + q4 + e) = __builtin_bit_cast(uint16_t, (__bf16)val[e]);
                            f32x4 one[1] = {val};
                            apply_act(P.act(), one);
                            val = one[0];
                        }
                        const int64_t oi = (int64_t)p * P.ldy + q4;
                        const int64_t ri = (int64_t)p * P.ldr + q4;
                        if (y_f32) {
                            float* yp = static_cast<float*>(P.y) + oi;
                            const float* rp = static_cast<const float*>(P.res);
                            if (vec_ok) {
                                if (RES32 && res_pre) val += rpre[RES32 ? mi : 0][RES32 ? cc : 0][RES32 ? pass : 0];
                                else if (rp) val += *as_global(reinterpret_cast<const f32x4*>(rp + ri));
                                *as_global(reinterpret_cast<f32x4*>(yp)) = val;
                            } else {
#pragma unroll
                                for (int e = 0; e < 4; ++e)
                                    if (q4 + e < N) *as_global(yp + e) = val[e] + (rp ? *as_global(rp + ri + e) : 0.f);
                            }
                        } else {
                            uint16_t* yp = static_cast<uint16_t*>(P.y) + oi;
                            const uint16_t* rp = static_cast<const uint16_t*>(P.res);
                            if (P.res_f32 && rp) {      // fp32 residual stream into a bf16 output
                                const float* rf = static_cast<const float*>(P.res);
                                if (RES32 && res_pre) val += rpre[RES32 ? mi : 0][RES32 ? cc : 0][RES32 ? pass : 0];
                                else if (vec_ok) val += *as_global(reinterpret_cast<const f32x4*>(rf + ri));
                                else
#pragma unroll
                                    for (int e = 0; e < 4; ++e)
                                        if (q4 + e < N) val[e] += *as_global(rf + ri + e);
                                rp = nullptr;
                            }
                            if (vec_ok) {
                                if (rp) {
                                    const u32x2 rv = *as_global(reinterpret_cast<const u32x2*>(rp + ri));
                                    val[0] += bf16lo_to_f32(rv[0]); val[1] += bf16hi_to_f32(rv[0]);
                                    val[2] += bf16lo_to_f32(rv[1]); val[3] += bf16hi_to_f32(rv[1]);
                                }
                                bf16x4 o;
#pragma unroll
                                for (int e = 0; e < 4; ++e) o[e] = (__bf16)val[e];
                                if (sig)   // device-scope store: read by tiles of this launch on other XCDs
                                    __hip_atomic_store(reinterpret_cast<uint64_t*>(yp), __builtin_bit_cast(uint64_t, o), __ATOMIC_RELAXED,
                                                       __HIP_MEMORY_SCOPE_AGENT);
                                else
                                    *as_global(reinterpret_cast<bf16x4*>(yp)) = o;
                            } else {
#pragma unroll
                                for (int e = 0; e < 4; ++e)
                                    if (q4 + e < N) {
                                        const float f = val[e] + (rp ? bf16_to_f32(*as_global(rp + ri + e)) : 0.f);
                                        *as_global(yp + e) = __builtin_bit_cast(uint16_t, (__bf16)f);
                                    }
                            }
                        }
                    }
                }
            }
            __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
            __builtin_amdgcn_wave_barrier();
        }
    }
    if (rec && tid == 0 && readers_before == P.readers - 1) DepRecord<DeviceMem>::clear(rec);
    // ---- tell the tiles that wait for this one: every wave's stores have completed at device
    // scope (vmcnt counts a device-scope store until it is visible there), then one flag add, or
    // the nonce in this column tile's word
    if (sig && P.nonce) {
        uint64_t* const w = reinterpret_cast<uint64_t*>(sig) + tm * (DEP_RECORD / 8);
        if (tid == 0) DepRecord<DeviceMem>::open(w, tn);
        wait_vmcnt<0>();
        __syncthreads();
        if (tid == 0) DepRecord<DeviceMem>::publish(w, tn, P.nonce);
    } else if (sig) {
        wait_vmcnt<0>();
        __syncthreads();
        if (tid == 0) __hip_atomic_fetch_add(sig + tm, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    }
}

template <int BM, int BN, int BK, int WGM, int WGN, int STAGES, bool GEGLU, bool GUARD, bool RES32, class Ext>
__global__ __launch_bounds__(64 * WGM * WGN, (gemm_min_waves<BM, BN, BK, WGM, WGN, STAGES>())) void gemm_kernel(const GemmGroup g, const Ext ext) {
    constexpr int NW = WGM * WGN;
    __shared__ u32x4 lds[gemm_lds_chunks<BM, BN, BK, WGM, WGN, STAGES>()];
    GemmProblem P;
    int tile, zero_n;
    int32_t* zero_ptr;
    const bool any = gemm_pick_tile(g, tile, P, zero_n, zero_ptr);
    // flags of the next dependent launch, a few words per workgroup: nothing reads them before this kernel ends
    for (int i = blockIdx.x * (64 * NW) + threadIdx.x; i < zero_n; i += (int)gridDim.x * (64 * NW)) zero_ptr[i] = 0;
    if (!any) return;
    if constexpr (BN > DOWN_BN && std::is_same_v<Ext, GemmPlain>) {
        if (P.signal) {
            gemm_tile<BM, DOWN_BN, BK, WGM * WGN / 2, 2, down_stages<BM, BN, BK, STAGES>(), false, GUARD, false>(P, tile, lds, ext);
            return;
        }
    }
    gemm_tile<BM, BN, BK, WGM, WGN, STAGES, GEGLU, GUARD, RES32>(P, tile, lds, ext);
}

}  // namespace sd
