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
// dz and its column sums.  256 columns and ROWS rows a workgroup: a lane has four columns, a wavefront every fourth row.  The sums of a
// workgroup's rows go to partials[row block], those of the blocks are added up by sum_partials.
// dz is rounded to bf16, which is what the matrix cores multiply (the sums are of what it was before); its rows are Np elements
// long, N rounded up to a multiple of 8, with zeros behind N.
// ---------------------------------------------------------------------------------------
constexpr int DZ_ROWS = 64;
template <class D, bool STORE, bool SUMS>
__global__ __launch_bounds__(256) void dz_kernel(const D* __restrict__ dy, const uint16_t* __restrict__ z, int act, uint16_t* __restrict__ dz, float* __restrict__ partials, int M, int N, int Np) {
    __shared__ f32x4 sh[3 * 64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int c = (blockIdx.y * 64 + lane) * 4;
    const int64_t r0 = (int64_t)blockIdx.x * DZ_ROWS + wave;
    const int64_t r1 = min((int64_t)M, ((int64_t)blockIdx.x + 1) * DZ_ROWS);
    const bool whole = c + 4 <= N;
    f32x4 sum = {0.f, 0.f, 0.f, 0.f};
    if (c < Np)
#pragma unroll 4
        for (int64_t r = r0; r < r1; r += 4) {
            f32x4 g = {0.f, 0.f, 0.f, 0.f}, v = g;
            const D* const dr = dy + r * N + c;
            const __bf16* const zr = reinterpret_cast<const __bf16*>(z) + r * N + c;
            if (whole) {
                g = load4(dr);
                if (z) v = load4(zr);
            } else {
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (c + e < N) {
                        g[e] = (float)dr[e];
                        if (z) v[e] = (float)zr[e];
                    }
            }
            if (z)
#pragma unroll
                for (int e = 0; e < 4; ++e) g[e] *= act_slope(act, v[e]);
            if (SUMS) sum += g;
            if (STORE) store4(reinterpret_cast<__bf16*>(dz) + r * Np + c, g);
        }
    if (SUMS) {
        if (wave) sh[(wave - 1) * 64 + lane] = sum;
        __syncthreads();
        if (wave == 0) {
#pragma unroll
            for (int w = 0; w < 3; ++w) sum += sh[w * 64 + lane];
            float* const out = partials + (int64_t)blockIdx.x * N + c;
            if (whole) store4(out, sum);
            else
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (c + e < N) out[e] = sum[e];
        }
    }
}

// out[i] = sum over s of parts[s n + i], in order; n % 4 == 0
template <class T>
__global__ __launch_bounds__(256) void sum_parts_kernel(const float* __restrict__ parts, int S, T* __restrict__ out, int64_t n) {
    const int64_t i = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 4;
    if (i >= n) return;
    f32x4 a = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
    for (int s = 0; s < S; ++s) a += load4(parts + s * n + i);
    store4(out + i, a);
}
static int launch_sum_parts(const float* parts, int S, void* out, bool f32, int64_t n, hipStream_t stream) {
    if (n == 0 || SD_DRY_RUN("sum parts; ")) return SD_OK;
    const dim3 grid((unsigned)((n / 4 + 255) / 256));
    if (f32) hipLaunchKernelGGL((sum_parts_kernel<float>), grid, dim3(256), 0, stream, parts, S, static_cast<float*>(out), n);
    else hipLaunchKernelGGL((sum_parts_kernel<__bf16>), grid, dim3(256), 0, stream, parts, S, static_cast<__bf16*>(out), n);
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

// Parts that the reduction of a backward product is cut into: as many as give every CU two tiles, none shorter than 256, and as many
// problems as a launch holds.  Their sums meet in fp32, in order.
constexpr int BWD_BM = 128, BWD_BN = 128;
static int bwd_parts(int64_t rows, int64_t cols, int64_t depth) {
    const int64_t tiles = ((rows + BWD_BM - 1) / BWD_BM) * ((cols + BWD_BN - 1) / BWD_BN);
    const int64_t parts = std::min<int64_t>(512 / std::max<int64_t>(tiles, 1), depth / 256);
    return (int)std::max<int64_t>(1, std::min<int64_t>(parts, GEMM_MAX_PROBLEMS));
}
static size_t bwd_parts_bytes(int64_t rows, int64_t cols, int64_t depth) {
    const int s = bwd_parts(rows, cols, depth);
    return s > 1 ? (size_t)s * rows * cols * 4 : 0;
}
// out [rows, cols] = P^T Q (PT) or P Q over `depth`; p [depth, rows] or [rows, depth], q [depth, cols]
template <bool PT>
static int bwd_product(const uint16_t* p, int64_t ldp, const uint16_t* q, int64_t ldq, void* out, bool out_f32, int rows, int cols, int depth, float* parts, hipStream_t stream) {
    const int S = bwd_parts(rows, cols, depth);
    const int steps = (depth + 63) / 64;
    GemmGroup g;
    memset(&g, 0, sizeof(g));
    for (int i = 0; i < S; ++i) {
        const int s0 = (int)((int64_t)steps * i / S), s1 = (int)((int64_t)steps * (i + 1) / S);
        GemmProblem& P = g.p[g.n++];
        P.p0 = p + (PT ? (int64_t)s0 * 64 * ldp : (int64_t)s0 * 64);
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
    int rc = launch_ext<BWD_BM, BWD_BN, 2, 2, 2, false>(g, depth % 64 != 0, GemmTransposed<PT, true>{}, stream);
    if (rc || S == 1) return rc;
    return launch_sum_parts(parts, S, out, out_f32, (int64_t)rows * cols, stream);
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
    size_t dz, sums, parts;
    BwdWs(int64_t M, int64_t N, int64_t K) {
        dz = (size_t)M * ((N + 7) & ~7ll) * 2;
        sums = (size_t)((M + DZ_ROWS - 1) / DZ_ROWS) * N * 4;
        parts = std::max(bwd_parts_bytes(M, K, N), bwd_parts_bytes(N, K, M));
    }
    size_t total() const { return round_up(dz, 256) + round_up(sums, 256) + round_up(parts, 256) + 256; }
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
    if (M == 0 || N == 0) {        // sums over nothing
        if (dx && M > 0 && (rc = launch_sum_parts(nullptr, 0, dx, false, (int64_t)M * K, s))) return rc;
        if (dW && N > 0 && (rc = launch_sum_parts(nullptr, 0, dW, dw_dtype == SD_F32, (int64_t)N * K, s))) return rc;
        return dbias && N > 0 ? launch_sum_partials(nullptr, 0, dbias, N, nullptr, 0, s) : SD_OK;
    }
    SD_REQUIRE(dy && (!dW || x) && (!dx || W), SD_EINVAL, "linear_bwd: dy, x or W is null");
    SD_REQUIRE(act == SD_ACT_NONE || z, SD_EINVAL, "linear_bwd: an activation needs z");
    if (!dx && !dW && !dbias) return SD_OK;
    const size_t need = sd_linear_bwd_workspace_bytes(M, N, K);
    SD_REQUIRE(ws && ws_bytes >= need && (reinterpret_cast<uintptr_t>(ws) & 255u) == 0, SD_EWORKSPACE, "linear_bwd: workspace of %zu bytes, need %zu, 256-byte aligned", ws_bytes, need);
    const BwdWs b(M, N, K);
    Workspace w(ws, ws_bytes);
    uint16_t* const dzbuf = static_cast<uint16_t*>(w.take(b.dz));
    float* const sums = static_cast<float*>(w.take(b.sums));
    float* const parts = static_cast<float*>(w.take(b.parts));
    const uint16_t* const zin = act == SD_ACT_NONE ? nullptr : z;
    const int Np = (N + 7) & ~7;
    // dz is dy itself where nothing changes it on the way
    const bool plain = !zin && y_dtype == SD_BF16 && Np == N;
    const bool store = (dx || dW) && !plain;
    if (store || dbias) {
        if (!SD_DRY_RUN("dz%s%s; ", store ? "" : " sums only", dbias ? "" : " no sums")) {
            const dim3 grid((unsigned)((M - 1) / DZ_ROWS + 1), (Np + 255) / 256);
            auto run = [&](auto* t) {
                using D = std::remove_pointer_t<decltype(t)>;
                const D* const d = static_cast<const D*>(dy);
                if (store && dbias) hipLaunchKernelGGL((dz_kernel<D, true, true>), grid, dim3(256), 0, s, d, zin, act, dzbuf, sums, M, N, Np);
                else if (store) hipLaunchKernelGGL((dz_kernel<D, true, false>), grid, dim3(256), 0, s, d, zin, act, dzbuf, sums, M, N, Np);
                else hipLaunchKernelGGL((dz_kernel<D, false, true>), grid, dim3(256), 0, s, d, zin, act, dzbuf, sums, M, N, Np);
            };
            if (y_dtype == SD_F32) run(static_cast<float*>(nullptr));
            else run(static_cast<__bf16*>(nullptr));
            SD_HIP_CHECK(hipGetLastError());
        }
        if (dbias && (rc = launch_sum_partials(sums, (M - 1) / DZ_ROWS + 1, dbias, N, nullptr, 0, s))) return rc;
    }
    const uint16_t* const dz = plain ? static_cast<const uint16_t*>(dy) : dzbuf;
    if (dx && (rc = bwd_product<false>(dz, Np, W, K, dx, false, M, K, N, parts, s))) return rc;
    if (dW && (rc = bwd_product<true>(dz, Np, x, K, dW, dw_dtype == SD_F32, N, K, M, parts, s))) return rc;
    return SD_OK;
}
