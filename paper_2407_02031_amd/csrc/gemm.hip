// The launches of the grouped projection kernel (gemm_tile.hpp): which tiles a group takes, and the flags that its
// dependent tiles wait for.
#include "gemm_tile.hpp"

namespace sd {

template <int BM, int BN, int BK, int WGM, int WGN, int STAGES, bool GEGLU, bool RES32>
static int launch_cfg(GemmGroup& g, bool guard, hipStream_t stream) {
    constexpr int BN_OUT = GEGLU ? BN / 2 : BN;
    int total = 0;
    g.n_lead = 0;
    for (int i = 0; i < g.n; ++i) {
        GemmProblem& P = g.p[i];
        P.tiles_m = (P.Mp + BM - 1) / BM;
        P.tiles_n = P.signal ? (P.N + (BN < DOWN_BN ? BN : DOWN_BN) - 1) / (BN < DOWN_BN ? BN : DOWN_BN) : (P.N + BN_OUT - 1) / BN_OUT;
        P.tile_begin = total;
        P.readers = P.tiles_n;
        g.first_tile[i] = total;
        total += P.tiles_m * P.tiles_n;
        if (P.signal) g.n_lead = total;
        P.wait_need = (P.K1 + (BN < DOWN_BN ? BN : DOWN_BN) - 1) / (BN < DOWN_BN ? BN : DOWN_BN);   // column tiles of the producer, whose N is this problem's K1
    }
    g.total_tiles = total;
    if (total == 0) return SD_OK;
    // A few tiles of longer K loops behind the producers' (text keys / values in a q, k, v launch) are dealt round-robin like those: in
    // one XCD's range they held up its other tiles (7904x1920x640 with 20 text tiles: every XCD was done after 26 us, that one after 34).  How few makes
    // no difference that could be measured (two blocks, none / up to 6 / 12.5 / 25 / 50 % of the tiles: 2 x 3952 x 640 589 581 582 582 583, 2 x 1024 x 1280 + 64
    // 519 518 514 512 514, 4 x 1200 x 640 + 32 422 418 418 420 417).
    int front = 0;
    for (int i = 0; i < g.n && (g.p[i].signal || g.p[i].K0 > g.p[g.n - 1].K0); ++i) front = g.p[i].tile_begin + g.p[i].tiles_m * g.p[i].tiles_n;
    if (front - g.n_lead <= total / 8) g.n_lead = front;
    if (SD_DRY_RUN("gemm %dx%d/%d waves/%d stages%s%s%s%s%s; ", BM, BN, WGM * WGN, STAGES, GEGLU ? " geglu" : "", RES32 ? " res32" : "", guard ? " guard" : "",
                   !g.p[0].signal ? "" : g.p[0].nonce ? " records" : " flags", dry_detail(", %d problems", g.n)))
        return SD_OK;
    if (guard)
        hipLaunchKernelGGL((gemm_kernel<BM, BN, BK, WGM, WGN, STAGES, GEGLU, true, RES32, GemmPlain>), dim3(g.n_lead + ((total - g.n_lead + 7) & ~7)), dim3(64 * WGM * WGN), 0, stream, g, GemmPlain{});
    else
        hipLaunchKernelGGL((gemm_kernel<BM, BN, BK, WGM, WGN, STAGES, GEGLU, false, RES32, GemmPlain>), dim3(g.n_lead + ((total - g.n_lead + 7) & ~7)), dim3(64 * WGM * WGN), 0, stream, g, GemmPlain{});
    SD_HIP_CHECK(hipGetLastError());
    return SD_OK;
}

template <int BM, int BN, int BK, int WGM, int WGN, int STAGES>
static int launch_res(GemmGroup& g, const GemmChoice& c, hipStream_t stream) {
    if (c.res32) return launch_cfg<BM, BN, BK, WGM, WGN, STAGES, false, true>(g, c.guard, stream);
    return launch_cfg<BM, BN, BK, WGM, WGN, STAGES, false, false>(g, c.guard, stream);
}

// Which kernel, from the problems' sizes alone.
GemmChoice gemm_choice(const GemmGroup& g) {
    bool geglu = false;   // a GEGLU group: GEGLU problems plus, possibly, the plain down-projections they wait for
    bool guard = false;
    int maxN = 0;
    double lead = 0;      // down-projection tiles of 128 rows: workgroups too, ahead of the others
    double depth = 0;     // K, summed over those tiles
    long t128 = 0, t256 = 0;   // workgroup tiles of 128 and 256 rows x 128 output columns, down-projections aside
    int gM = 0, gF = 0, gK = 0, gr = 0;   // the GEGLU problems: rows in all, largest F, K and rank
    bool res32 = false;   // some problem adds an fp32 residual: take the kernel that prefetches it
    int n_main = 0;       // problems that are not down-projections
    bool mixed = false;   // ... of different widths or depths
    int N0 = 0, K0 = 0;
    for (int i = 0; i < g.n; ++i) {
        const GemmProblem& P = g.p[i];
        if (P.geglu_F > 0) geglu = true;
        if (P.Mp == 0 || P.N == 0) continue;
        if ((P.K0 & 63) || (P.K1 & 63)) guard = true;
        if (P.res && P.res_f32) res32 = true;
        if (P.N > maxN) maxN = P.N;
        if (P.signal) {
            lead += (double)((P.Mp + 127) / 128) * ((P.N + DOWN_BN - 1) / DOWN_BN);
            continue;
        }
        mixed = mixed || (n_main++ && (P.N != N0 || P.K0 != K0));
        N0 = P.N, K0 = P.K0;
        if (P.geglu_F > 0) {
            gM += P.Mp;
            gF = P.N > gF ? P.N : gF;
            gK = P.K0 > gK ? P.K0 : gK;
            gr = P.K1 > gr ? P.K1 : gr;
        }
        const long tiles = (long)((P.Mp + 127) / 128) * ((P.N + 127) / 128);
        t128 += tiles;
        t256 += (long)((P.Mp + 255) / 256) * ((P.N + 127) / 128);
        depth += (double)tiles * P.K0;
    }
    auto take = [&](GemmTiles t) { return GemmChoice{t, guard, res32}; };
    // Tile choice.  What a tile costs per 64 deep step is its operand bytes (a CU takes in 100-125 GB/s
    // from L2 whatever the ring depth) or its MFMAs, whichever is longer, and the launch takes as long
    // as its most loaded CU; so: the largest tiles that still give every CU the same number of them.
    // Times below are single projections of rank 64, us, measured on one machine.
    const double meanK = t128 ? depth / t128 : 0;
    // GEGLU: geglu_tiles (128 columns of W are 64 of the output)
    if (geglu) switch (geglu_tiles(gM, gF, gK, gr, false)) {
        case GEGLU_64x64_3STAGES: return take(GEMM_GEGLU_64x128_3STAGES);
        case GEGLU_64x64: return take(GEMM_GEGLU_64x128);
        case GEGLU_256x128: return take(GEMM_GEGLU_256x256);
        default: return take(GEMM_GEGLU_128x128);
        }
    // Down-projections (N = rank <= 64) alone: 64x64 tiles, 5-stage ring.
    if (maxN <= 64) return take(GEMM_64x64);
    if (t128 < 512) {
        // at most one 128x128 tile per CU, and most CUs have one: that tile with a deep ring, one
        // workgroup per CU (2048x1280x5120: 42.0, 53.7 with 64x128 tiles, of which 64 CUs get two)
        if (t128 > 128 && gemm_one_round(t128, (long)lead)) return take(GEMM_128x128_ONE_ROUND);
        // more than that (the down-projection's tiles count), but at most one of 256x128 per CU, and no short K loop: those
        // (8192x640x2560: 41.1, 48.2 with 128x128 tiles; 4757x1280x1280: 26.4, 33.1 with 64x128;
        // 6000x640x2560 34.5, 44.5 with 128x128 tiles; at K = 640 the ramps of the larger tile lose: 24.1 against 21.0)
        if (t128 > 128 && t256 + lead / 2 <= 256 && meanK >= 1024) return take(GEMM_256x128_ONE_ROUND);
        // few tiles: 64x128 spreads them over more CUs, two workgroups on a CU at most: three ring stages
        if (t128 <= 128) return take(GEMM_64x128_3STAGES);
        // up to three on a CU where the K loop is short (8192x640x640: 17.3, 18.3 with 128x128)
        if (t128 > 256 && meanK < 1024) return take(GEMM_64x128);
    }
    // One large plain projection with a long K loop (no launch of the transformer block: the
    // 8192 x 4096 x 4096 yardstick takes 220, 245 at 256x128, 260 at 128x128; 8192x8192x2048 + 64 256, 284, 290; but
    // 16384x1280x5120 + 64, five of these tiles wide, 254, 217, 236).  Not for grouped
    // launches: the q/k/v group with its short text-context problems loses a third.
    if (!res32 && n_main == 1 && t256 >= 512 && meanK >= 2048) return take(GEMM_256x256);
    // 128x128 tiles, two workgroups per CU.  Of eight 32x64 wavefronts where problems of different sizes share the launch (q, k,
    // v transposed, text keys): their tiles load the CUs unevenly, and one that has a CU to itself is faster with more
    // wavefronts (attention blocks, us, four / eight: 4 x 3952 tokens of 640 channels with text keys + 64 106.7 / 100.4, 2 x 988 of
    // 1280 + 16 85.6 / 79.8, 2 x 4096 of 320 + 8 109.8 / 100.5, 4 x 3952 of 640 + 32 275.4 / 279.2; 80 of them 0.91 to 1.014)
    if (mixed && !res32) return take(GEMM_128x128_8WAVES);
    // ... of four 64x64 otherwise (4757x1280x1280: 25.9, 33.1 with 64x128, 26.9 with eight wavefronts; the segments of a multi-adapter
    // call: 8 x 4096 of 640 channels 45.0 / 45.6, 2999,2221,1552,1847,895 of 1280 48.6 / 50.7, of 320 up to 12 % the other way)
    return take(GEMM_128x128);
}

int launch_gemm_group(GemmGroup& g, hipStream_t stream) {
    SD_REQUIRE(g.n >= 1 && g.n <= GEMM_MAX_PROBLEMS, SD_EINVAL, "gemm group: %d problems", g.n);
    bool geglu = false;
    for (int i = 0; i < g.n; ++i) geglu = geglu || g.p[i].geglu_F > 0;
    for (int i = 0; i < g.n; ++i) {
        const GemmProblem& P = g.p[i];
        SD_REQUIRE(!P.linear(), SD_EINVAL, "gemm problem %d: a linear layer", i);
        SD_REQUIRE((P.geglu_F > 0) == geglu || P.signal, SD_EINVAL, "gemm group mixes GEGLU and plain problems");
        SD_REQUIRE(P.Mp >= 0 && P.N >= 0 && P.K0 > 0 && P.K0 % 8 == 0 && P.K1 >= 0 && P.K1 % 8 == 0, SD_EINVAL,
                   "gemm problem %d: bad sizes M=%d N=%d K0=%d K1=%d", i, P.Mp, P.N, P.K0, P.K1);
        SD_REQUIRE(P.p0 && P.q0 && P.y && (P.K1 == 0 || (P.p1 && P.q1)), SD_EINVAL, "gemm problem %d: null operand", i);
        SD_REQUIRE(P.ldp0 % 8 == 0 && P.ldq0 % 8 == 0 && (P.K1 == 0 || (P.ldp1 % 8 == 0 && P.ldq1 % 8 == 0)), SD_EINVAL,
                   "gemm problem %d: leading dimensions must be multiples of 8", i);
        // lane offsets inside a tile are 32-bit byte offsets
        const int64_t span = 256 + (P.geglu_F > 0 ? P.geglu_F : 0);
        SD_REQUIRE(P.ldp0 > 0 && P.ldq0 > 0 && P.ldp0 * 256 < (1ll << 31) && P.ldq0 * span < (1ll << 31) &&
                       (P.K1 == 0 || (P.ldp1 > 0 && P.ldq1 > 0 && P.ldp1 * 256 < (1ll << 31) && P.ldq1 * span < (1ll << 31))),
                   SD_EINVAL, "gemm problem %d: leading dimension out of range", i);
        if (P.signal) {
            SD_REQUIRE(i == 0 || g.p[i - 1].signal, SD_EINVAL, "gemm group: signalling problem %d after a plain one", i);
            SD_REQUIRE(!P.y_f32 && !P.res && !P.wait && P.N % 4 == 0 && P.ldy % 4 == 0 && P.geglu_F == 0, SD_EINVAL,
                       "gemm problem %d: a signalling problem stores plain bf16 rows", i);
        }
        SD_REQUIRE(!P.nonce || (P.signal ? P.N <= DEP_PRODUCERS * DOWN_BN : (P.wait && !P.wait_cols && P.K1 <= DEP_PRODUCERS * DOWN_BN)), SD_EINVAL,
                   "gemm problem %d: what a dependency record does not hold", i);
        SD_REQUIRE(!P.wait || (P.K1 > 0 && g.p[0].signal), SD_EINVAL, "gemm problem %d waits but the group has no producer", i);
    }
    // drop empty problems
    int w = 0;
    for (int i = 0; i < g.n; ++i)
        if (g.p[i].Mp > 0 && g.p[i].N > 0) { if (w != i) g.p[w] = g.p[i]; ++w; }
    g.n = w;
    if (w == 0) return SD_OK;
    const GemmChoice c = gemm_choice(g);
    switch (c.tiles) {
    case GEMM_GEGLU_64x128_3STAGES: return launch_cfg<64, 128, 64, 2, 2, 3, true, false>(g, c.guard, stream);
    case GEMM_GEGLU_64x128: return launch_cfg<64, 128, 64, 2, 2, 2, true, false>(g, c.guard, stream);
    case GEMM_GEGLU_256x256: return launch_cfg<256, 256, 64, 4, 2, 2, true, false>(g, c.guard, stream);
    case GEMM_GEGLU_128x128: return launch_cfg<128, 128, 64, 2, 2, 2, true, false>(g, c.guard, stream);
    case GEMM_64x64: return launch_cfg<64, 64, 64, 2, 2, 5, false, false>(g, c.guard, stream);
    case GEMM_128x128_ONE_ROUND: return launch_res<128, 128, 64, 4, 2, 4>(g, c, stream);
    case GEMM_256x128_ONE_ROUND: return launch_res<256, 128, 64, 4, 2, 3>(g, c, stream);
    case GEMM_64x128_3STAGES: return launch_res<64, 128, 64, 2, 2, 3>(g, c, stream);
    case GEMM_64x128: return launch_res<64, 128, 64, 2, 2, 2>(g, c, stream);
    case GEMM_256x256: return launch_cfg<256, 256, 64, 4, 2, 2, false, false>(g, c.guard, stream);
    case GEMM_128x128_8WAVES: return launch_cfg<128, 128, 64, 4, 2, 2, false, false>(g, c.guard, stream);
    default: return launch_res<128, 128, 64, 2, 2, 2>(g, c, stream);
    }
}

__global__ void clear_flags_kernel(int32_t* p, int n) {
    const int i = blockIdx.x * blockDim.x + threadIdx.x;
    if (i < n) p[i] = 0;
}
int launch_clear_flags(int32_t* p, int n, hipStream_t stream) {
    if (n <= 0 || SD_DRY_RUN("clear; ")) return SD_OK;
    hipLaunchKernelGGL(clear_flags_kernel, dim3((n + 255) / 256), dim3(256), 0, stream, p, n);
    SD_HIP_CHECK(hipGetLastError());
    return SD_OK;
}
int gemm_dep_timeouts(long long* count) {
    unsigned long long v = 0;
    SD_HIP_CHECK(hipMemcpyFromSymbol(&v, HIP_SYMBOL(g_gemm_dep_timeouts), sizeof(v)));
    *count = (long long)v;
    return SD_OK;
}

}  // namespace sd
