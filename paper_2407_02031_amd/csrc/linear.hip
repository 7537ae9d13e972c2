// A linear layer with bias, activation and residual, and its backward pass.
//
//   z = x W^T + bias,  y = act(z) + residual
//   dz = dy act'(z):  dx = dz W,  dW = dz^T x,  dbias = sum_m dz
//
// The products run on the projections' tiles (gemm_tile.hpp): forward with the activation in the epilogue; backward with operands
// whose rows are the reduction's, which the transposing LDS read turns on the way into the registers, so that nothing is
// transposed in memory.  dz is formed once, in front of the products, by a kernel that sums its columns in fp32 too.
#include "gemm_tile.hpp"
#include "rows.hpp"

#include <string.h>
#include <algorithm>

namespace sd {

// ---------------------------------------------------------------------------------------
// dz and its column sums.  512 columns and DZ_ROWS rows a workgroup: a lane has eight columns, a wavefront every fourth row.  The sums
// of a workgroup's rows go to sums[row block] (of the one row block of a short dy, to the result itself).
// dz is rounded to bf16, which is what the matrix cores multiply (the sums are of what it was before); its rows are Np elements
// long, N rounded up to a multiple of 8, with zeros behind N.
// ---------------------------------------------------------------------------------------
constexpr int DZ_ROWS = 64, DZ_COLS = 512;
template <class D, bool STORE, bool SUMS>
__global__ __launch_bounds__(256) void dz_kernel(const D* __restrict__ dy, const uint16_t* __restrict__ z, int act, uint16_t* __restrict__ dz, float* __restrict__ sums, int M, int N, int Np) {
    __shared__ f32x8 sh[3 * 64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int c = blockIdx.y * DZ_COLS + lane * 8;
    const int64_t r0 = (int64_t)blockIdx.x * DZ_ROWS + wave;
    const int64_t r1 = min((int64_t)M, ((int64_t)blockIdx.x + 1) * DZ_ROWS);
    const bool whole = c + 8 <= N;
    const f32x4 zero = {0.f, 0.f, 0.f, 0.f};
    f32x8 sum = {zero, zero};
    auto slope = [&](f32x8 g, const f32x8& v) {
        if (z)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                g.lo[e] *= act_slope(act, v.lo[e]);
                g.hi[e] *= act_slope(act, v.hi[e]);
            }
        if (SUMS) {
            sum.lo += g.lo;
            sum.hi += g.hi;
        }
        return g;
    };
    // A row's last piece, where eight do not divide it, begins earlier, at N - 8: what it has in common with its neighbour's is written
    // twice, the same, and counted in the neighbour's sums alone.
    const int at = whole ? c : N - 8;
    if (N >= 8 && c < Np) {
#pragma unroll 4
        for (int64_t r = r0; r < r1; r += 4) {
            f32x8 v = {zero, zero};
            if (z) v = load8(reinterpret_cast<const __bf16*>(z) + r * N + at);
            const f32x8 g = slope(load8(dy + r * N + at), v);
            if (STORE) {
                store8(reinterpret_cast<__bf16*>(dz) + r * Np + at, g);
                if (!whole)
                    for (int e = N; e < Np; ++e) dz[r * Np + e] = 0;
            }
        }
    } else if (c < Np) {
        for (int64_t r = r0; r < r1; r += 4) {
            f32x8 g = {zero, zero}, v = g;
#pragma unroll
            for (int e = 0; e < 7; ++e)
                if (e < N) {
                    const float d = (float)dy[r * N + e], w = z ? bf16_to_f32(z[r * N + e]) : 0.f;
                    if (e < 4) g.lo[e & 3] = d, v.lo[e & 3] = w;
                    else g.hi[e & 3] = d, v.hi[e & 3] = w;
                }
            g = slope(g, v);
            if (STORE) store8(reinterpret_cast<__bf16*>(dz) + r * Np, g);
        }
    }
    if (SUMS) {
        if (wave) sh[(wave - 1) * 64 + lane] = sum;
        __syncthreads();
        if (wave == 0) {
#pragma unroll
            for (int w = 0; w < 3; ++w) {
                sum.lo += sh[w * 64 + lane].lo;
                sum.hi += sh[w * 64 + lane].hi;
            }
            float* const out = sums + (int64_t)blockIdx.x * N + c;
            if (whole) {
                store4(out, sum.lo);
                store4(out + 4, sum.hi);
            } else {
                const int first = N >= 8 ? N - 8 : 0;
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    if (first + e >= c && first + e < N) out[first - c + e] = e < 4 ? sum.lo[e & 3] : sum.hi[e & 3];
            }
        }
    }
}

// ---------------------------------------------------------------------------------------
// What is left in parts: dx, dW (as many fp32 matrices as their reductions were cut into) and dbias (a row for every
// row block of dz), each added up in order, in one launch.  256 threads: 1024 elements of a matrix, or 64 columns of dbias.
// ---------------------------------------------------------------------------------------
struct Parts {
    const float* parts;
    void* out;
    int64_t n;            // elements
    int32_t count, f32;
    int32_t wgs;
};
struct PartSums {
    Parts m[2];
    const float* sums;
    float* dbias;
    int32_t blocks, N;
};
template <class T>
__device__ __forceinline__ void sum_parts(const Parts& p, int wg) {
    const int64_t i = ((int64_t)wg * 256 + threadIdx.x) * 4;
    if (i >= p.n) return;
    f32x4 a = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
    for (int s = 0; s < p.count; ++s) a += load4(p.parts + s * p.n + i);
    store4(static_cast<T*>(p.out) + i, a);
}
__global__ __launch_bounds__(256) void part_sums_kernel(const PartSums a) {
    int wg = blockIdx.x;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        if (wg < a.m[i].wgs) {
            if (a.m[i].f32) sum_parts<float>(a.m[i], wg);
            else sum_parts<__bf16>(a.m[i], wg);
            return;
        }
        wg -= a.m[i].wgs;
    }
    __shared__ float sh[3][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, c = wg * 64 + lane;
    float s = 0.f;
    if (c < a.N)
#pragma unroll 8
        for (int b = wave; b < a.blocks; b += 4) s += a.sums[(int64_t)b * a.N + c];
    if (wave) sh[wave - 1][lane] = s;
    __syncthreads();
    if (wave == 0 && c < a.N) a.dbias[c] = s + sh[0][lane] + sh[1][lane] + sh[2][lane];
}
static Parts parts_of(const float* parts, void* out, bool f32, int64_t n, int count) { return Parts{parts, out, n, count, f32, (int32_t)((n / 4 + 255) / 256)}; }
static int launch_part_sums(PartSums& a, hipStream_t stream) {
    const int64_t wgs = (int64_t)a.m[0].wgs + a.m[1].wgs + (a.dbias ? (a.N + 63) / 64 : 0);
    if (wgs == 0 || SD_DRY_RUN("part sums; ")) return SD_OK;
    hipLaunchKernelGGL(part_sums_kernel, dim3((unsigned)wgs), dim3(256), 0, stream, a);
    SD_HIP_CHECK(hipGetLastError());
    return SD_OK;
}

// ---------------------------------------------------------------------------------------
// products
// ---------------------------------------------------------------------------------------
template <int BM, int BN, int WGM, int WGN, int STAGES, bool RES32, class Ext>
static int launch_ext(GemmGroup& g, bool guard, const Ext& ext, hipStream_t stream) {
    int total = 0;
    for (int i = 0; i < g.n; ++i) {
        GemmProblem& P = g.p[i];
        P.tiles_m = (P.Mp + BM - 1) / BM;
        P.tiles_n = (P.N + BN - 1) / BN;
        P.tile_begin = total;
        g.first_tile[i] = total;
        total += P.tiles_m * P.tiles_n;
    }
    g.total_tiles = total;
    if (SD_DRY_RUN("gemm %s %dx%d/%d waves/%d stages%s%s%s; ", Ext::act ? "act" : Ext::pt ? "dW" : "dx", BM, BN, WGM * WGN, STAGES, RES32 ? " res32" : "", guard ? " guard" : "",
                   dry_detail(", %d problems", g.n)))
        return SD_OK;
    const dim3 grid((total + 7) & ~7), block(64 * WGM * WGN);
    if (guard) hipLaunchKernelGGL((gemm_kernel<BM, BN, 64, WGM, WGN, STAGES, false, true, RES32, Ext>), grid, block, 0, stream, g, ext);
    else hipLaunchKernelGGL((gemm_kernel<BM, BN, 64, WGM, WGN, STAGES, false, false, RES32, Ext>), grid, block, 0, stream, g, ext);
    SD_HIP_CHECK(hipGetLastError());
    return SD_OK;
}
template <int BM, int BN, int WGM, int WGN, int STAGES>
static int launch_act(GemmGroup& g, const GemmChoice& c, const GemmAct& ext, hipStream_t stream) {
    if (c.res32) return launch_ext<BM, BN, WGM, WGN, STAGES, true>(g, c.guard, ext, stream);
    return launch_ext<BM, BN, WGM, WGN, STAGES, false>(g, c.guard, ext, stream);
}

// ---------------------------------------------------------------------------------------
// Both products of a backward pass in one launch: the tiles of the one fill the CUs that those of the other leave.  Every XCD gets
// an eighth of each product's tiles, in order, those with more steps first.
// ---------------------------------------------------------------------------------------
template <int BM, int BN, int WGM, int WGN, int STAGES, bool GUARD>
__global__ __launch_bounds__(64 * WGM * WGN, (gemm_min_waves<BM, BN, 64, WGM, WGN, STAGES>())) void gemm_bwd_kernel(const GemmGroup g, const int dw_from, const int dw_to) {
    __shared__ u32x4 lds[gemm_lds_chunks<BM, BN, 64, WGM, WGN, STAGES>()];
    int j = blockIdx.x >> 3, pi = 0, tiles = 0, per = 0;
    for (; pi < g.n; ++pi) {
        tiles = (pi + 1 < g.n ? g.first_tile[pi + 1] : g.total_tiles) - g.first_tile[pi];
        per = (tiles + 7) >> 3;
        if (j < per) break;
        j -= per;
    }
    const int t = (int)(blockIdx.x & 7) * per + j;
    if (pi == g.n || t >= tiles) return;
    ProblemRegs r;
    load_problem(g.p[pi], r);
    asm volatile("" : "+s"(r.a), "+s"(r.b), "+s"(r.c), "+s"(r.d), "+s"(r.e));
    const GemmProblem P = problem_of(r);
    if (pi >= dw_from && pi < dw_to) gemm_tile<BM, BN, 64, WGM, WGN, STAGES, false, GUARD, false>(P, P.tile_begin + t, lds, GemmTransposed<true, true>{});
    else gemm_tile<BM, BN, 64, WGM, WGN, STAGES, false, GUARD, false>(P, P.tile_begin + t, lds, GemmTransposed<false, true>{});
}

// Into how many parts the reductions are cut: so that none is longer than what a workgroup's share of all steps is, two workgroups a CU,
// but none shorter than BWD_STEPS, and no more problems than a launch holds.
constexpr int BWD_BM = 128, BWD_BN = 128, BWD_STEPS = 4;
// (From the sizes alone, as for both products: a gradient's bits do not depend on which others are wanted.)
struct BwdPlan {
    int dx, dw;          // parts
    BwdPlan(int64_t M, int64_t N, int64_t K) {
        auto tiles = [](int64_t r, int64_t c) { return ((r + BWD_BM - 1) / BWD_BM) * ((c + BWD_BN - 1) / BWD_BN); };
        const int64_t sx = (N + 63) / 64, sw = (M + 63) / 64;
        const int64_t all = tiles(M, K) * sx + tiles(N, K) * sw;
        const int64_t share = std::max<int64_t>(all / 512, BWD_STEPS);
        auto parts = [&](int64_t steps) { return (int)std::min<int64_t>(std::max<int64_t>(steps / share, 1), GEMM_MAX_PROBLEMS / 2); };
        dx = parts(sx);
        dw = parts(sw);
    }
};
// out [rows, cols] = P^T Q (pt) or P Q over `depth`; p [depth, rows] or [rows, depth], q [depth, cols]
static void push_product(GemmGroup& g, bool pt, const uint16_t* p, int64_t ldp, const uint16_t* q, int64_t ldq, void* out, bool out_f32, int rows, int cols, int depth, int S, float* parts) {
    const int steps = (depth + 63) / 64;
    for (int i = 0; i < S; ++i) {
        const int s0 = (int)((int64_t)steps * i / S), s1 = (int)((int64_t)steps * (i + 1) / S);
        GemmProblem& P = g.p[g.n++];
        P.p0 = p + (pt ? (int64_t)s0 * 64 * ldp : (int64_t)s0 * 64);
        P.ldp0 = ldp;
        P.q0 = q + (int64_t)s0 * 64 * ldq;
        P.ldq0 = ldq;
        P.Mp = rows;
        P.N = cols;
        P.K0 = std::min(depth, s1 * 64) - s0 * 64;
        P.alpha = 1.f;
        P.ldy = cols;
        P.y = S > 1 ? static_cast<void*>(parts + (int64_t)i * rows * cols) : out;
        P.y_f32 = S > 1 || out_f32;
    }
}
template <int BM, int BN, int WGM, int WGN, int STAGES>
static int launch_bwd(GemmGroup& g, int dw_from, int dw_to, bool guard, hipStream_t stream) {
    int total = 0, per = 0;
    for (int i = 0; i < g.n; ++i) {
        GemmProblem& P = g.p[i];
        P.tiles_m = (P.Mp + BM - 1) / BM;
        P.tiles_n = (P.N + BN - 1) / BN;
        P.tile_begin = total;
        g.first_tile[i] = total;
        total += P.tiles_m * P.tiles_n;
        per += (P.tiles_m * P.tiles_n + 7) / 8;
    }
    g.total_tiles = total;
    if (SD_DRY_RUN("gemm bwd %dx%d/%d waves/%d stages%s%s; ", BM, BN, WGM * WGN, STAGES, guard ? " guard" : "", dry_detail(", %d of dW, %d of dx", dw_to - dw_from, g.n - (dw_to - dw_from))))
        return SD_OK;
    const dim3 grid(8 * per), block(64 * WGM * WGN);
    if (guard) hipLaunchKernelGGL((gemm_bwd_kernel<BM, BN, WGM, WGN, STAGES, true>), grid, block, 0, stream, g, dw_from, dw_to);
    else hipLaunchKernelGGL((gemm_bwd_kernel<BM, BN, WGM, WGN, STAGES, false>), grid, block, 0, stream, g, dw_from, dw_to);
    SD_HIP_CHECK(hipGetLastError());
    return SD_OK;
}

// ---------------------------------------------------------------------------------------
// Few rows (one token's, a guidance pair's): bound by the weights, which come in once.  A workgroup has 16 columns, whose rows of W its
// wavefronts bring straight into the registers as MFMA operands, every NW-th step of 32 each; their sums meet in LDS.
// ---------------------------------------------------------------------------------------
template <int NW, int MB>
__global__ __launch_bounds__(64 * NW) void linear_rows_kernel(const uint16_t* __restrict__ x, const uint16_t* __restrict__ W, const uint16_t* __restrict__ bias, int act, const void* res,
                                                              void* y, int f32, uint16_t* __restrict__ z, int M, int N, int K) {
    constexpr int U = 8;             // steps in flight
    __shared__ f32x4 sh[NW * MB * 64];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int l16 = lane & 15, quad = lane >> 4;
    const int n0 = blockIdx.x * 16;
    const uint16_t* const wr = W + (int64_t)min(n0 + l16, N - 1) * K + quad * 8;
    const uint16_t* xr[MB];
    f32x4 acc[MB];
#pragma unroll
    for (int m = 0; m < MB; ++m) {
        xr[m] = x + (int64_t)min(m * 16 + l16, M - 1) * K + quad * 8;
        acc[m] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
    const int steps = (K + 31) / 32;
    const u32x4 none = {0u, 0u, 0u, 0u};
    for (int s0 = wave; s0 < steps; s0 += NW * U) {
        u32x4 wf[U], xf[U][MB];
#pragma unroll
        for (int i = 0; i < U; ++i) {
            const int k = (s0 + i * NW) * 32;
            const bool in = k + quad * 8 < K;         // (a chunk of eight is whole or not there)
            wf[i] = in ? *reinterpret_cast<const u32x4*>(wr + k) : none;
#pragma unroll
            for (int m = 0; m < MB; ++m) xf[i][m] = in ? *reinterpret_cast<const u32x4*>(xr[m] + k) : none;
        }
#pragma unroll
        for (int i = 0; i < U; ++i)
#pragma unroll
            for (int m = 0; m < MB; ++m)
                acc[m] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, wf[i]), __builtin_bit_cast(bf16x8, xf[i][m]), acc[m], 0, 0, 0);
    }
#pragma unroll
    for (int m = 0; m < MB; ++m) sh[(wave * MB + m) * 64 + lane] = acc[m];
    __syncthreads();
    if (wave >= MB) return;
    // ---- wavefront m finishes block m: a lane has four columns of one row
    const int row = wave * 16 + l16, col = n0 + quad * 4;
    f32x4 v[1] = {sh[wave * 64 + lane]};
#pragma unroll
    for (int w = 1; w < NW; ++w) v[0] += sh[(w * MB + wave) * 64 + lane];
    if (row >= M || col >= N) return;
    const int64_t at = (int64_t)row * N + col;
    const __bf16* const bb = reinterpret_cast<const __bf16*>(bias);
    if (col + 4 <= N) {
        if (bias) v[0] += load4(bb + col);
        if (z) store4(reinterpret_cast<__bf16*>(z) + at, v[0]);
        apply_act(act, v);
        if (res) v[0] += f32 ? load4(static_cast<const float*>(res) + at) : load4(static_cast<const __bf16*>(res) + at);
        if (f32) store4(static_cast<float*>(y) + at, v[0]);
        else store4(static_cast<__bf16*>(y) + at, v[0]);
        return;
    }
    if (bias)
#pragma unroll
        for (int e = 0; e < 3; ++e)
            if (col + e < N) v[0][e] += (float)bb[col + e];
    const f32x4 pre = v[0];
    apply_act(act, v);
#pragma unroll
    for (int e = 0; e < 3; ++e)
        if (col + e < N) {
            if (z) reinterpret_cast<__bf16*>(z)[at + e] = (__bf16)pre[e];
            const float r = !res ? 0.f : f32 ? static_cast<const float*>(res)[at + e] : (float)static_cast<const __bf16*>(res)[at + e];
            if (f32) static_cast<float*>(y)[at + e] = v[0][e] + r;
            else static_cast<__bf16*>(y)[at + e] = (__bf16)(v[0][e] + r);
        }
}
constexpr int LINEAR_ROWS = 32;       // rows that this kernel takes
template <int NW>
static int launch_rows(const uint16_t* x, const uint16_t* W, const uint16_t* bias, int act, const void* res, void* y, int f32, uint16_t* z, int M, int N, int K, hipStream_t stream) {
    if (SD_DRY_RUN("linear rows %d/%d waves; ", M > 16 ? 32 : 16, NW)) return SD_OK;
    const dim3 grid((N + 15) / 16), block(64 * NW);
    if (M <= 16) hipLaunchKernelGGL((linear_rows_kernel<NW, 1>), grid, block, 0, stream, x, W, bias, act, res, y, f32, z, M, N, K);
    else hipLaunchKernelGGL((linear_rows_kernel<NW, 2>), grid, block, 0, stream, x, W, bias, act, res, y, f32, z, M, N, K);
    SD_HIP_CHECK(hipGetLastError());
    return SD_OK;
}

static int linear_sizes(const char* who, int M, int N, int K, int act, int y_dtype) {
    SD_REQUIRE(M >= 0 && N >= 0, SD_EINVAL, "%s: M=%d N=%d", who, M, N);
    SD_REQUIRE(K > 0 && K % 8 == 0, SD_EUNSUPPORTED, "%s: K=%d is not a positive multiple of 8", who, K);
    SD_REQUIRE(K < (1 << 22) && N < (1 << 22), SD_EUNSUPPORTED, "%s: N=%d K=%d (below 2^22)", who, N, K);
    SD_REQUIRE((M / 64 + 1ll) * (N / 64 + 1) < (1ll << 30) && (M / 128 + 1ll) * (K / 128 + 1) < (1ll << 26), SD_EUNSUPPORTED, "%s: M=%d N=%d K=%d", who, M, N, K);
    SD_REQUIRE(act >= SD_ACT_NONE && act <= SD_ACT_RELU, SD_EINVAL, "%s: activation %d", who, act);
    SD_REQUIRE(y_dtype == SD_BF16 || y_dtype == SD_F32, SD_EINVAL, "%s: y_dtype=%d", who, y_dtype);
    return SD_OK;
}
// what sd_linear_bwd carves out of its workspace
struct BwdWs {
    size_t dz, sums, dx_parts, dw_parts;
    BwdWs(int64_t M, int64_t N, int64_t K) {
        dz = (size_t)M * ((N + 7) & ~7ll) * 2;
        sums = (size_t)((M + DZ_ROWS - 1) / DZ_ROWS) * N * 4;
        const BwdPlan p(M, N, K);
        dx_parts = p.dx > 1 ? (size_t)p.dx * M * K * 4 : 0;
        dw_parts = p.dw > 1 ? (size_t)p.dw * N * K * 4 : 0;
    }
    size_t total() const { return round_up(dz, 256) + round_up(sums, 256) + round_up(dx_parts, 256) + round_up(dw_parts, 256) + 256; }
};

}  // namespace sd

using namespace sd;

extern "C" int sd_linear_fwd(const uint16_t* x, const uint16_t* W, const uint16_t* bias, int32_t act, const void* residual, void* y, int32_t y_dtype, uint16_t* z,
                             int32_t M, int32_t N, int32_t K, void* stream) {
    int rc = linear_sizes("linear_fwd", M, N, K, act, y_dtype);
    if (rc || M == 0 || N == 0) return rc;
    SD_REQUIRE(x && W && y, SD_EINVAL, "linear_fwd: x, W or y is null");
    SD_REQUIRE(aligned16(x) && aligned16(W) && aligned16(bias) && aligned16(residual) && aligned16(y) && aligned16(z), SD_EINVAL, "linear_fwd: pointers must be 16-byte aligned");
    hipStream_t s = static_cast<hipStream_t>(stream);
    if (M <= LINEAR_ROWS) return K > 2048 ? launch_rows<16>(x, W, bias, act, residual, y, y_dtype == SD_F32, z, M, N, K, s) : launch_rows<8>(x, W, bias, act, residual, y, y_dtype == SD_F32, z, M, N, K, s);
    GemmGroup g;
    memset(&g, 0, sizeof(g));
    g.n = 1;
    GemmProblem& P = g.p[0];
    P.p0 = x; P.ldp0 = K;
    P.q0 = W; P.ldq0 = K;
    P.bias = bias;
    P.res = residual; P.ldr = N; P.res_f32 = y_dtype == SD_F32;
    P.y = y; P.ldy = N; P.y_f32 = y_dtype == SD_F32;
    P.Mp = M; P.N = N; P.K0 = K; P.alpha = 1.f;
    if (act == SD_ACT_NONE && !z) return gemm16_takes(g) ? launch_gemm16(g, s) : launch_gemm_group(g, s);
    const GemmAct ext{z, act};
    const GemmChoice c = gemm_choice(g);
    switch (c.tiles) {
    case GEMM_64x64: return launch_ext<64, 64, 2, 2, 5, false>(g, c.guard, ext, s);
    case GEMM_64x128_3STAGES: return launch_act<64, 128, 2, 2, 3>(g, c, ext, s);
    case GEMM_64x128: return launch_act<64, 128, 2, 2, 2>(g, c, ext, s);
    case GEMM_128x128_ONE_ROUND: return launch_act<128, 128, 4, 2, 4>(g, c, ext, s);
    case GEMM_256x128_ONE_ROUND: return launch_act<256, 128, 4, 2, 3>(g, c, ext, s);
    case GEMM_256x256: return launch_ext<256, 256, 4, 2, 2, false>(g, c.guard, ext, s);
    default: return launch_act<128, 128, 2, 2, 2>(g, c, ext, s);
    }
}

extern "C" size_t sd_linear_bwd_workspace_bytes(int32_t M, int32_t N, int32_t K) {
    if (M <= 0 || N <= 0 || K <= 0) return 256;
    return BwdWs(M, N, K).total();
}

extern "C" int sd_linear_bwd(const void* dy, int32_t y_dtype, const uint16_t* x, const uint16_t* W, const uint16_t* z, int32_t act, uint16_t* dx, void* dW, int32_t dw_dtype,
                             float* dbias, int32_t M, int32_t N, int32_t K, void* ws, size_t ws_bytes, void* stream) {
    int rc = linear_sizes("linear_bwd", M, N, K, act, y_dtype);
    if (rc) return rc;
    SD_REQUIRE(dw_dtype == SD_BF16 || dw_dtype == SD_F32, SD_EINVAL, "linear_bwd: dw_dtype=%d", dw_dtype);
    SD_REQUIRE(aligned16(dy) && aligned16(x) && aligned16(W) && aligned16(z) && aligned16(dx) && aligned16(dW) && aligned16(dbias), SD_EINVAL,
               "linear_bwd: pointers must be 16-byte aligned");
    hipStream_t s = static_cast<hipStream_t>(stream);
    PartSums left;
    memset(&left, 0, sizeof(left));
    if (M == 0 || N == 0) {        // sums over nothing
        if (dx) left.m[0] = parts_of(nullptr, dx, false, (int64_t)M * K, 0);
        if (dW) left.m[1] = parts_of(nullptr, dW, dw_dtype == SD_F32, (int64_t)N * K, 0);
        left.dbias = dbias;
        left.N = N;
        return launch_part_sums(left, s);
    }
    SD_REQUIRE(dy && (!dW || x) && (!dx || W), SD_EINVAL, "linear_bwd: dy, x or W is null");
    SD_REQUIRE(act == SD_ACT_NONE || z, SD_EINVAL, "linear_bwd: an activation needs z");
    if (!dx && !dW && !dbias) return SD_OK;
    const size_t need = sd_linear_bwd_workspace_bytes(M, N, K);
    SD_REQUIRE(ws && ws_bytes >= need && (reinterpret_cast<uintptr_t>(ws) & 255u) == 0, SD_EWORKSPACE, "linear_bwd: workspace of %zu bytes, need %zu, 256-byte aligned", ws_bytes, need);
    const BwdWs b(M, N, K);
    const BwdPlan plan(M, N, K);
    Workspace w(ws, ws_bytes);
    uint16_t* const dzbuf = static_cast<uint16_t*>(w.take(b.dz));
    float* const sums = static_cast<float*>(w.take(b.sums));
    float* const dx_parts = static_cast<float*>(w.take(b.dx_parts));
    float* const dw_parts = static_cast<float*>(w.take(b.dw_parts));
    const uint16_t* const zin = act == SD_ACT_NONE ? nullptr : z;
    const int Np = (N + 7) & ~7, blocks = (M - 1) / DZ_ROWS + 1;
    // dz is dy itself where nothing changes it on the way
    const bool plain = !zin && y_dtype == SD_BF16 && Np == N;
    const bool store = (dx || dW) && !plain;
    if ((store || dbias) && !SD_DRY_RUN("dz%s%s; ", store ? "" : " sums only", dbias ? "" : " no sums")) {
        const dim3 grid((unsigned)blocks, (Np + DZ_COLS - 1) / DZ_COLS);
        float* const to = blocks == 1 ? dbias : sums;
        auto run = [&](auto* t) {
            using D = std::remove_pointer_t<decltype(t)>;
            const D* const d = static_cast<const D*>(dy);
            if (store && dbias) hipLaunchKernelGGL((dz_kernel<D, true, true>), grid, dim3(256), 0, s, d, zin, act, dzbuf, to, M, N, Np);
            else if (store) hipLaunchKernelGGL((dz_kernel<D, true, false>), grid, dim3(256), 0, s, d, zin, act, dzbuf, to, M, N, Np);
            else hipLaunchKernelGGL((dz_kernel<D, false, true>), grid, dim3(256), 0, s, d, zin, act, dzbuf, to, M, N, Np);
        };
        if (y_dtype == SD_F32) run(static_cast<float*>(nullptr));
        else run(static_cast<__bf16*>(nullptr));
        SD_HIP_CHECK(hipGetLastError());
    }
    if (dbias && blocks > 1) {
        left.sums = sums;
        left.dbias = dbias;
        left.blocks = blocks;
        left.N = N;
    }
    if (dx || dW) {
        const uint16_t* const dz = plain ? static_cast<const uint16_t*>(dy) : dzbuf;
        GemmGroup g;
        memset(&g, 0, sizeof(g));
        // the longer parts first
        const bool dw_first = dW && (!dx || ((M + 63) / 64) / plan.dw >= ((N + 63) / 64) / plan.dx);
        auto push_dw = [&] {
            if (dW) push_product(g, true, dz, Np, x, K, dW, dw_dtype == SD_F32, N, K, M, plan.dw, dw_parts);
        };
        if (dw_first) push_dw();
        const int dx_from = g.n;
        if (dx) push_product(g, false, dz, Np, W, K, dx, false, M, K, N, plan.dx, dx_parts);
        const int dx_to = g.n;
        if (!dw_first) push_dw();
        const bool guard = (dW && M % 64 != 0) || (dx && N % 64 != 0);
        if ((rc = launch_bwd<BWD_BM, BWD_BN, 2, 2, 2>(g, dw_first ? 0 : dx_to, dw_first ? dx_from : g.n, guard, s))) return rc;
        if (dx && plan.dx > 1) left.m[0] = parts_of(dx_parts, dx, false, (int64_t)M * K, plan.dx);
        if (dW && plan.dw > 1) left.m[1] = parts_of(dw_parts, dW, dw_dtype == SD_F32, (int64_t)N * K, plan.dw);
    }
    return launch_part_sums(left, s);
}
