// A linear layer, and a gated one, of rows in 8 bits with scales (fp8.hpp).
//
//   y = act(x W^T + bias) + residual;      gated: y = (x Wv^T + bv) act(x Wg^T + bg), in bf16, fp32, or 8 bits again
//
// On the tiles of gemm_cols.hpp: the scaled MFMA multiplies at twice the rate of a bf16 one and reads half the bytes.
//
// Measured: 8192 x 4096 x 4096 bf16 out 119 us (2.3 PFLOP/s; the library's 102), 8192 x 5120 x 1280 67.6 (1.6; the library's 72); gated with SiLU, 8192 x 5120 x 1280, 101 to bf16, 102 to 8 bits (2.1; the library's
// product alone 107), of which the main loops take 79.  1976 x 1280 x 5120 onto fp32 32.2.  One row, 5120 x 1280 gated to 8 bits 11.0 to 11.3, 1280 x 5120 onto fp32 6.5.
// With sums asked for whole (widened operands): 8192 x 5120 x 1280 106 to bf16, gated 194 to bf16, 207 to 8 bits; 1976 x 1280 x 5120 to bf16 31 for 25.
#include "gemm_cols.hpp"

#include <string.h>

namespace sd {

static int linear8_check(const char* who, const uint8_t* x, const uint8_t* x_scales, int64_t x_lds, const uint8_t* W, const uint8_t* w_scales, int64_t w_lds, int act, int M, int N, int64_t w_rows, int K) {
    SD_REQUIRE(M >= 0 && N >= 0, SD_EINVAL, "%s: M=%d N=%d", who, M, N);
    SD_REQUIRE(M < (1 << 27) && N < (1 << 22), SD_EUNSUPPORTED, "%s: M=%d N=%d (M below 2^27, N below 2^22)", who, M, N);
    SD_REQUIRE(act >= SD_ACT_NONE && act <= SD_ACT_RELU, SD_EINVAL, "%s: activation %d", who, act);
    SD_REQUIRE(K > 0 && K % 16 == 0 && K < (1 << 22), SD_EUNSUPPORTED, "%s: K=%d is not a positive multiple of 16 below 2^22", who, K);
    SD_REQUIRE(!cols_too_many(M, w_rows, false), SD_EUNSUPPORTED, "%s: M=%d N=%d (2^22 tiles of 64 x 64 and more)", who, M, N);
    if (M == 0 || N == 0) return SD_OK;
    const int rc = fp8_check(who, "x", x, x_scales, x_lds, M, K);
    return rc ? rc : fp8_check(who, "W", W, w_scales, w_lds, w_rows, K);
}
static ColsProblem problem8(const uint8_t* x, const uint8_t* x_scales, int64_t x_lds, const uint8_t* W, const uint8_t* w_scales, int64_t w_lds, const uint16_t* bias, int act, void* y, int M, int N, int K) {
    ColsProblem P;
    memset(&P, 0, sizeof(P));
    P.p = x; P.ps = x_scales; P.ldps = x_lds;
    P.q = W; P.qs = w_scales; P.ldqs = w_lds;
    P.bias = bias; P.act = act; P.y = y;
    P.M = M; P.N = N; P.Kb = K;
    return P;
}

// Tiles (gemm_cols.hpp's rule).  It takes 50 to 72 launches each 0.6 % (plain), 0.4 % (gated), 0 % (to 8 bits), 1.1 % (y in fp32) and 0.6 % (gated, y in fp32) longer in the mean than the fastest of these tiles.
static const ColsTile PLAIN8[] = {{256, 256, 256, 0.f, 7.1f, 1.134f, 7.1f, 1.134f}, {128, 256, 256, 0.f, 5.7f, 0.62f, 5.7f, 0.62f}, {256, 128, 256, 0.f, 5.5f, 0.618f, 5.5f, 0.618f},
                                  {128, 192, 256, 0.f, 5.2f, 0.625f, 5.2f, 0.625f}, {96, 128, 256, 1.f, 3.f, 0.522f, 3.f, 0.522f}, {128, 128, 512, 0.f, 6.6f, 0.995f, 3.7f, 0.724f},
                                  {64, 128, 512, 0.4f, 3.4f, 0.702f, 3.2f, 0.324f}, {64, 64, 512, 1.2f, 2.1f, 0.436f, 2.2f, 0.193f}};
static const ColsTile GATED8[] = {{256, 256, 256, 0.f, 5.7f, 1.4f, 5.7f, 1.4f}, {128, 256, 256, 0.f, 4.9f, 0.744f, 4.9f, 0.744f}, {256, 128, 256, 0.f, 5.f, 0.675f, 5.f, 0.675f},
                                  {128, 128, 512, 0.f, 4.7f, 0.994f, 3.7f, 0.762f}, {64, 128, 512, 1.4f, 2.7f, 0.655f, 2.1f, 0.381f}, {64, 64, 512, 0.f, 2.8f, 0.528f, 3.5f, 0.306f}};
static const ColsTile GATED8_TO_8[] = {{256, 256, 256, 0.f, 6.8f, 1.32f, 6.8f, 1.32f}, {128, 256, 256, 0.f, 5.4f, 0.735f, 5.4f, 0.735f}, {64, 256, 256, 0.7f, 4.2f, 0.626f, 4.2f, 0.626f}};
static const ColsTile WIDE8[] = {{128, 256, 256, 0.f, 13.3f, 1.243f, 13.3f, 1.243f}, {128, 192, 256, 0.f, 11.1f, 1.072f, 11.1f, 1.072f}, {96, 128, 256, 0.f, 7.9f, 0.615f, 7.9f, 0.615f},
                                 {64, 128, 512, 2.1f, 8.2f, 0.918f, 3.6f, 0.491f}, {64, 64, 512, 1.9f, 4.5f, 0.617f, 2.7f, 0.363f}};
static const ColsTile GATED_WIDE8[] = {{128, 128, 512, 2.f, 5.3f, 1.445f, 2.6f, 1.027f}, {128, 128, 256, 0.3f, 5.1f, 0.722f, 5.1f, 0.722f}, {64, 128, 512, 2.3f, 3.4f, 0.875f, 2.2f, 0.503f},
                                       {64, 64, 512, 2.5f, 2.7f, 0.514f, 1.6f, 0.323f}};

// y in 8 bits of sums that the caller wants whole.  (6 % off 240 launches of 65 to 8192 rows in the mean, and the fastest of these each time.)
static const ColsTile GATED_WIDE8_TO_8[] = {{128, 256, 256, 0.f, 6.4f, 1.29f, 6.4f, 1.29f}, {64, 256, 256, 0.4f, 5.1f, 0.745f, 5.1f, 0.745f}, {32, 256, 256, 0.8f, 3.9f, 0.575f, 3.9f, 0.575f}};

// Few rows: straight from the weights where that is one workgroup a CU.  With widened operands, whose tiles are slower, with more rows and columns a workgroup too.  (us, these kernels / tiles:
// 32 x 1280 x 5120 7.7 / 10.6, 32 x 1280 x 1280 4.1 / 5.1, 64 x 1280 x 5120 10.3 / 11.1, but 128 of them 12.9 / 11.2; y in fp32 256 x 1280 x 1280 7.5 / 8.2, 128 of them 5.8 / 8.0; gated 64 x 1280 x 5120 12.8 / 17.1.)
enum FewRows { FEW_NONE, FEW_16x16, FEW_32x16, FEW_32x32, FEW_64x32 };
static FewRows few8_choose(bool gated, bool wide, int M, int N) {
    const int64_t r16 = (M + 15) / 16, r32 = (M + 31) / 32, r64 = (M + 63) / 64, c16 = (N + 15) / 16, c32 = (N + 31) / 32;
    if (r16 * c16 <= 256) return FEW_16x16;
    if (r32 * c16 <= 256) return FEW_32x16;
    if (wide && r32 * c32 <= 256) return FEW_32x32;
    return !gated && wide && r64 * c32 <= 256 ? FEW_64x32 : FEW_NONE;
}
template <bool GATED>
static int launch_few8(const ColsProblem& P, bool wide, bool& taken, hipStream_t s) {
    const FewRows few = few8_choose(GATED, wide, P.M, P.N);
    taken = few != FEW_NONE;
    switch (few) {
    case FEW_16x16: return launch_few<true, GATED, 1, 1, GATED ? 2 : 4>(P, s);
    case FEW_32x16: return launch_few<true, GATED, 2, 1, GATED ? 2 : 4>(P, s);
    case FEW_32x32: return launch_few<true, GATED, 2, 2, GATED ? 2 : 3>(P, s);
    case FEW_64x32:
        if constexpr (!GATED) return launch_few<true, false, 4, 2, 2>(P, s);
        break;
    default: break;
    }
    return SD_OK;
}
// y in 8 bits by way of fp32, in two launches: where a block's columns lie in several workgroups (few rows, smaller tiles), which a long reduction makes up for.  (us, one launch / two, of which the second
// is 6, and what the rule adds for it, with its start, 9: 64 x 1280 x 5120 30.2 / 18, 256 of them 32.5 / 22; 64 x 5120 x 1280 11.6 / 13.)
// Each as it is launched, up to 64 rows widened.  The one launch of these draws the weights through one CU for each 128 columns, the slower the more of them there are (us, one launch as taken and as measured, two as measured: one row 5120 x 1280
// 12.6 / 11.9, 9.2; 5120 x 2560 20.7 / 20.8, 12.6; 5120 x 5120 36.9 / 35.1, 19.2; 10240 x 5120 43.3 / 40.9, 30.6; 3 rows 15552 x 4144 42.1 / 42.8, 29.4).
static bool gated8_one_widened(int M, int N) { return M <= 64 && (int64_t)((M + 31) / 32) * ((N + FP8_BLOCK - 1) / FP8_BLOCK) <= 256; }
static bool gated8_two_launches(int M, int N, int K) {
    float one, two;
    const float steps = (float)((K + 127) / 128);
    if (gated8_one_widened(M, N)) one = 4.5f + (0.65f + 0.004f * (float)((N + FP8_BLOCK - 1) / FP8_BLOCK)) * steps;
    else cols_choose(GATED8_TO_8, M, 2ll * N, K, one);
    switch (few8_choose(true, true, M, N)) {        // (within 15 % of these kernels at 5 to 40 steps)
    case FEW_16x16: two = 3.f + 0.18f * steps; break;
    case FEW_32x16: two = 3.f + 0.24f * steps; break;
    case FEW_32x32: two = 3.5f + 0.3f * steps; break;
    default:
        if (M <= 64) cols_choose(GATED_WIDE8, M, 2ll * N, K, two);
        else cols_choose(GATED8, M, 2ll * N, K, two);
    }
    return two + 9.f + (float)M * N * 2e-6f < one;
}
static int launch_gated8(ColsProblem& P, bool wide, hipStream_t s) {
    float us;
    if (wide)
        switch (cols_choose(GATED_WIDE8, P.M, 2ll * P.N, P.Kb, us)) {
        case 0: return launch_cols<COLS_FP8_WIDE, 128, 128, 2, 2, 2, true, false>(P, s);
        case 1: return launch_cols<COLS_FP8_WIDE, 128, 128, 2, 2, 3, true, false, 2>(P, s);
        case 2: return launch_cols<COLS_FP8_WIDE, 64, 128, 2, 2, 3, true, false>(P, s);
        default: return launch_cols<COLS_FP8_WIDE, 64, 64, 2, 1, 4, true, false, 2>(P, s);
        }
    switch (cols_choose(GATED8, P.M, 2ll * P.N, P.Kb, us)) {
    case 0: return launch_cols<COLS_FP8, 256, 256, 2, 4, 2, true, false>(P, s);
    case 1: return launch_cols<COLS_FP8, 128, 256, 2, 4, 3, true, false>(P, s);
    case 2: return launch_cols<COLS_FP8, 256, 128, 4, 2, 3, true, false>(P, s);
    case 3: return launch_cols<COLS_FP8, 128, 128, 2, 2, 2, true, false>(P, s);
    case 4: return launch_cols<COLS_FP8, 64, 128, 2, 2, 3, true, false>(P, s);
    default: return launch_cols<COLS_FP8, 64, 64, 2, 1, 4, true, false>(P, s);
    }
}

}  // namespace sd

using namespace sd;

extern "C" int sd_linear_fp8_fwd(const uint8_t* x, const uint8_t* x_scales, int64_t x_lds, const uint8_t* W, const uint8_t* w_scales, int64_t w_lds, const uint16_t* bias, int32_t act, const void* residual,
                                 void* y, int32_t y_dtype, int32_t M, int32_t N, int32_t K, void* stream) {
    const bool wide = y_dtype == SD_F32 || (act & SD_WHOLE_SUMS);
    act &= ~SD_WHOLE_SUMS;
    const int rc = linear8_check("linear_fp8_fwd", x, x_scales, x_lds, W, w_scales, w_lds, act, M, N, N, K);
    if (rc) return rc;
    SD_REQUIRE(y_dtype == SD_BF16 || y_dtype == SD_F32, SD_EINVAL, "linear_fp8_fwd: y_dtype=%d", y_dtype);
    if (M == 0 || N == 0) return SD_OK;
    SD_REQUIRE(y && aligned16(y) && aligned16(bias) && aligned16(residual), SD_EINVAL, "linear_fp8_fwd: y is null, or a pointer is not 16-byte aligned");
    for (const void* in : {static_cast<const void*>(x), static_cast<const void*>(x_scales), static_cast<const void*>(W), static_cast<const void*>(w_scales), static_cast<const void*>(bias)})
        SD_REQUIRE(y != in, SD_EINVAL, "linear_fp8_fwd: y in an input's place");
    ColsProblem P = problem8(x, x_scales, x_lds, W, w_scales, w_lds, bias, act, y, M, N, K);
    P.res = residual;
    P.y_f32 = y_dtype == SD_F32;
    hipStream_t s = static_cast<hipStream_t>(stream);
    bool taken;
    const int few = launch_few8<false>(P, wide, taken, s);
    if (taken) return few;
    float us;
    if (wide)
        switch (cols_choose(WIDE8, M, N, K, us)) {
        case 0: return launch_cols<COLS_FP8_WIDE, 128, 256, 2, 4, 3, false, false>(P, s);
        case 1: return launch_cols<COLS_FP8_WIDE, 128, 192, 4, 2, 3, false, false>(P, s);
        case 2: return launch_cols<COLS_FP8_WIDE, 96, 128, 1, 4, 3, false, false, 2>(P, s);
        case 3: return launch_cols<COLS_FP8_WIDE, 64, 128, 2, 2, 3, false, false, 2>(P, s);
        default: return launch_cols<COLS_FP8_WIDE, 64, 64, 2, 2, 4, false, false, 2>(P, s);
        }
    switch (cols_choose(PLAIN8, M, N, K, us)) {
    case 0: return launch_cols<COLS_FP8, 256, 256, 4, 2, 2, false, false>(P, s);
    case 1: return launch_cols<COLS_FP8, 128, 256, 2, 4, 3, false, false>(P, s);
    case 2: return launch_cols<COLS_FP8, 256, 128, 4, 2, 3, false, false>(P, s);
    case 3: return launch_cols<COLS_FP8, 128, 192, 4, 2, 3, false, false>(P, s);
    case 4: return launch_cols<COLS_FP8, 96, 128, 1, 4, 3, false, false>(P, s);
    case 5: return launch_cols<COLS_FP8, 128, 128, 2, 2, 2, false, false>(P, s);
    case 6: return launch_cols<COLS_FP8, 64, 128, 2, 2, 3, false, false>(P, s);
    default: return launch_cols<COLS_FP8, 64, 64, 2, 2, 4, false, false>(P, s);
    }
}

extern "C" size_t sd_gated_linear_fp8_workspace_bytes(int32_t M, int32_t N, int32_t K) {
    if (M <= 0 || N <= 0 || K <= 0 || M >= (1 << 27) || N >= (1 << 21) || !gated8_two_launches(M, N, K)) return 0;
    return round_up((size_t)M * N * 4, 256);
}

extern "C" int sd_gated_linear_fp8_fwd(const uint8_t* x, const uint8_t* x_scales, int64_t x_lds, const uint8_t* W, const uint8_t* w_scales, int64_t w_lds, const uint16_t* bias, int32_t act,
                                       void* y, int32_t y_dtype, uint8_t* y_scales, int64_t y_lds, int32_t M, int32_t N, int32_t K, void* ws, size_t ws_bytes, void* stream) {
    const bool whole = (act & SD_WHOLE_SUMS) != 0;
    act &= ~SD_WHOLE_SUMS;
    int rc = linear8_check("gated_linear_fp8_fwd", x, x_scales, x_lds, W, w_scales, w_lds, act, M, N, 2ll * N, K);
    if (rc) return rc;
    SD_REQUIRE(y_dtype == SD_BF16 || y_dtype == SD_F32 || y_dtype == SD_FP8, SD_EINVAL, "gated_linear_fp8_fwd: y_dtype=%d", y_dtype);
    SD_REQUIRE(N % 16 == 0 && N < (1 << 21), SD_EUNSUPPORTED, "gated_linear_fp8_fwd: N=%d is not a multiple of 16 below 2^21", N);
    if (M == 0 || N == 0) return SD_OK;
    SD_REQUIRE(y && aligned16(y) && aligned16(bias), SD_EINVAL, "gated_linear_fp8_fwd: y is null, or a pointer is not 16-byte aligned");
    for (const void* in : {static_cast<const void*>(x), static_cast<const void*>(x_scales), static_cast<const void*>(W), static_cast<const void*>(w_scales), static_cast<const void*>(bias)})
        SD_REQUIRE(y != in && (y_dtype != SD_FP8 || y_scales != in), SD_EINVAL, "gated_linear_fp8_fwd: y or its scales in an input's place");
    const bool out8 = y_dtype == SD_FP8;
    if (out8) {
        rc = fp8_check("gated_linear_fp8_fwd", "y", y, y_scales, y_lds, M, N);
        if (rc) return rc;
        SD_REQUIRE(y != y_scales, SD_EINVAL, "gated_linear_fp8_fwd: y's scales in y's place");
    }
    ColsProblem P = problem8(x, x_scales, x_lds, W, w_scales, w_lds, bias, act, y, M, N, K);
    P.y_f32 = y_dtype == SD_F32;
    hipStream_t s = static_cast<hipStream_t>(stream);
    bool taken;
    if (out8 && !gated8_two_launches(M, N, K)) {
        P.ys = y_scales;
        P.ldys = y_lds;
        // Up to 64 rows, where weights are all that counts, widened operands cost nothing (us, 32 x 256 widened / 64 x 256: one row 5120 x 1280 11.4 / 11.8, 10240 x 2560 21.1 / 21.4, 1280 x 2560 15.7 / 15.1)
        if (gated8_one_widened(M, N)) return launch_cols<COLS_FP8_WIDE, 32, 256, 1, 2, 3, true, true, 2>(P, s);
        float us;
        if (whole)
            switch (cols_choose(GATED_WIDE8_TO_8, M, 2ll * N, K, us)) {
            case 0: return launch_cols<COLS_FP8_WIDE, 128, 256, 4, 2, 3, true, true>(P, s);
            case 1: return launch_cols<COLS_FP8_WIDE, 64, 256, 2, 2, 3, true, true, 2>(P, s);
            default: return launch_cols<COLS_FP8_WIDE, 32, 256, 1, 2, 3, true, true, 2>(P, s);
            }
        switch (cols_choose(GATED8_TO_8, M, 2ll * N, K, us)) {
        case 0: return launch_cols<COLS_FP8, 256, 256, 4, 2, 2, true, true>(P, s);
        case 1: return launch_cols<COLS_FP8, 128, 256, 4, 2, 3, true, true>(P, s);
        default: return launch_cols<COLS_FP8, 64, 256, 2, 2, 3, true, true>(P, s);
        }
    }
    if (out8) {
        const size_t need = sd_gated_linear_fp8_workspace_bytes(M, N, K);
        SD_REQUIRE(ws && ws_bytes >= need && (reinterpret_cast<uintptr_t>(ws) & 255u) == 0, SD_EWORKSPACE, "gated_linear_fp8_fwd: workspace of %zu bytes, need %zu, 256-byte aligned", ws_bytes, need);
        P.y = ws;
        P.y_f32 = 1;
    }
    const bool wide = y_dtype == SD_F32 || whole || (out8 && M <= 64);
    rc = launch_few8<true>(P, y_dtype == SD_F32 || whole || out8, taken, s);
    // (to 8 bits widened up to 64 rows, as in one launch.  us, both launches, widened / not: one row 10240 x 5120 30.6 / 27.0, 5120 x 5120 19.9 / 18.7, 64 rows of them 36.1 / 36.2 and 22.3 / 21.5)
    if (!taken) rc = launch_gated8(P, wide, s);
    return rc || !out8 ? rc : launch_quantize(ws, true, static_cast<uint8_t*>(y), y_scales, y_lds, M, N, s);
}
