// A linear layer, and a gated one, of rows in 8 bits with scales (fp8.hpp).
//
//   y = act(x W^T + bias) + residual;      gated: y = (x Wv^T + bv) act(x Wg^T + bg), in bf16, fp32, or 8 bits again
//
// On the tiles of gemm_cols.hpp: the scaled MFMA multiplies at twice the rate of a bf16 one and reads half the bytes.
#include "gemm_cols.hpp"

#include <string.h>

namespace sd {

static int linear8_check(const char* who, const uint8_t* x, const uint8_t* x_scales, int64_t x_lds, const uint8_t* W, const uint8_t* w_scales, int64_t w_lds, int act, int M, int N, int64_t w_rows, int K) {
    SD_REQUIRE(M >= 0 && N >= 0, SD_EINVAL, "%s: M=%d N=%d", who, M, N);
    SD_REQUIRE(M < (1 << 27) && N < (1 << 22), SD_EUNSUPPORTED, "%s: M=%d N=%d (M below 2^27, N below 2^22)", who, M, N);
    SD_REQUIRE(act >= SD_ACT_NONE && act <= SD_ACT_RELU, SD_EINVAL, "%s: activation %d", who, act);
    SD_REQUIRE(K > 0 && K % 16 == 0 && K < (1 << 22), SD_EUNSUPPORTED, "%s: K=%d is not a positive multiple of 16 below 2^22", who, K);
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

}  // namespace sd

using namespace sd;

extern "C" int sd_linear_fp8_fwd(const uint8_t* x, const uint8_t* x_scales, int64_t x_lds, const uint8_t* W, const uint8_t* w_scales, int64_t w_lds, const uint16_t* bias, int32_t act, const void* residual,
                                 void* y, int32_t y_dtype, int32_t M, int32_t N, int32_t K, void* stream) {
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
    if (M <= 16) return launch_few<true, false, 1, 1, 4>(P, s);
    if (P.y_f32) return launch_cols<COLS_FP8_WIDE, 64, 128, 2, 2, 3, false, false>(P, s);
    if (M <= 512) return launch_cols<COLS_FP8, 64, 128, 2, 2, 3, false, false>(P, s);
    return launch_cols<COLS_FP8, 256, 256, 4, 2, 2, false, false>(P, s);
}

// few rows whose y goes out in 8 bits: y in fp32 first, as a block's columns lie in several workgroups
static bool gated8_few(int M) { return M <= 16; }
extern "C" size_t sd_gated_linear_fp8_workspace_bytes(int32_t M, int32_t N, int32_t K) {
    (void)K;
    if (M <= 0 || N <= 0 || !gated8_few(M) || N >= (1 << 22)) return 256;
    return round_up((size_t)M * N * 4, 256);
}

extern "C" int sd_gated_linear_fp8_fwd(const uint8_t* x, const uint8_t* x_scales, int64_t x_lds, const uint8_t* W, const uint8_t* w_scales, int64_t w_lds, const uint16_t* bias, int32_t act,
                                       void* y, int32_t y_dtype, uint8_t* y_scales, int64_t y_lds, int32_t M, int32_t N, int32_t K, void* ws, size_t ws_bytes, void* stream) {
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
    if (gated8_few(M)) {
        if (!out8) return launch_few<true, true, 1, 1, 2>(P, s);
        const size_t need = sd_gated_linear_fp8_workspace_bytes(M, N, K);
        SD_REQUIRE(ws && ws_bytes >= need && (reinterpret_cast<uintptr_t>(ws) & 255u) == 0, SD_EWORKSPACE, "gated_linear_fp8_fwd: workspace of %zu bytes, need %zu, 256-byte aligned", ws_bytes, need);
        P.y = ws;
        P.y_f32 = 1;
        rc = launch_few<true, true, 1, 1, 2>(P, s);
        return rc ? rc : launch_quantize(ws, true, static_cast<uint8_t*>(y), y_scales, y_lds, M, N, s);
    }
    if (out8) {
        P.ys = y_scales;
        P.ldys = y_lds;
        if (M <= 512) return launch_cols<COLS_FP8, 128, 256, 4, 2, 3, true, true>(P, s);
        return launch_cols<COLS_FP8, 256, 256, 4, 2, 2, true, true>(P, s);
    }
    if (P.y_f32) return launch_cols<COLS_FP8_WIDE, 64, 128, 2, 2, 3, true, false>(P, s);
    if (M <= 512) return launch_cols<COLS_FP8, 64, 128, 2, 2, 3, true, false>(P, s);
    return launch_cols<COLS_FP8, 256, 256, 4, 2, 2, true, false>(P, s);
}
