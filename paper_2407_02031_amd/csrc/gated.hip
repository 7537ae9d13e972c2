// A gated linear layer in bf16, as in training:
//
//   v = x Wv^T + bv,  g = x Wg^T + bg,  y = v act(g),  W = [Wv; Wg]
//
// Both projections, the activation and the product in one kernel (gemm_cols.hpp); v and g are kept in bf16 where the backward pass (linear.hip) wants them.
//
// Measured: 8192 x 5120 x 1280 with SiLU 188 us, 209 with v and g kept (252 MB of results; 1.0 to 1.1 PFLOP/s, the library's product alone 176).
#include "gemm_cols.hpp"

#include <string.h>

namespace sd {

// (gemm_cols.hpp's rule; it takes 48 launches 1 % longer in the mean than the fastest of these)
static const ColsTile GATED16[] = {{256, 256, 256, 0.f, 5.6f, 1.518f, 5.6f, 1.518f}, {128, 256, 256, 0.f, 5.1f, 0.816f, 5.1f, 0.816f}, {256, 128, 256, 0.f, 5.4f, 0.721f, 5.4f, 0.721f},
                                   {128, 128, 256, 0.f, 4.6f, 0.527f, 4.6f, 0.527f}, {64, 128, 512, 0.8f, 3.7f, 0.71f, 2.5f, 0.408f}, {64, 64, 512, 1.5f, 2.4f, 0.447f, 1.8f, 0.244f}};

}  // namespace sd

using namespace sd;

extern "C" int sd_gated_linear_fwd(const uint16_t* x, const uint16_t* W, const uint16_t* bias, int32_t act, void* y, int32_t y_dtype, uint16_t* z, int32_t M, int32_t N, int32_t K, void* stream) {
    SD_REQUIRE(M >= 0 && N >= 0, SD_EINVAL, "gated_linear_fwd: M=%d N=%d", M, N);
    SD_REQUIRE(K > 0 && K % 8 == 0, SD_EUNSUPPORTED, "gated_linear_fwd: K=%d is not a positive multiple of 8", K);
    SD_REQUIRE(M < (1 << 27) && N < (1 << 21) && K < (1 << 22), SD_EUNSUPPORTED, "gated_linear_fwd: M=%d N=%d K=%d (M below 2^27, N below 2^21, K below 2^22)", M, N, K);
    SD_REQUIRE(act >= SD_ACT_NONE && act <= SD_ACT_RELU, SD_EINVAL, "gated_linear_fwd: activation %d", act);
    SD_REQUIRE(y_dtype == SD_BF16 || y_dtype == SD_F32, SD_EINVAL, "gated_linear_fwd: y_dtype=%d", y_dtype);
    SD_REQUIRE(!cols_too_many(M, N, true), SD_EUNSUPPORTED, "gated_linear_fwd: M=%d N=%d (2^22 tiles of 64 x 64 and more)", M, N);
    if (M == 0 || N == 0) return SD_OK;
    SD_REQUIRE(x && W && y, SD_EINVAL, "gated_linear_fwd: x, W or y is null");
    SD_REQUIRE(aligned16(x) && aligned16(W) && aligned16(bias) && aligned16(y) && aligned16(z), SD_EINVAL, "gated_linear_fwd: pointers must be 16-byte aligned");
    SD_REQUIRE(y != x && y != W && y != bias && y != z && (!z || (z != x && z != W && z != bias)), SD_EINVAL, "gated_linear_fwd: y or z in an input's place");
    ColsProblem P;
    memset(&P, 0, sizeof(P));
    P.p = reinterpret_cast<const uint8_t*>(x);
    P.q = reinterpret_cast<const uint8_t*>(W);
    P.bias = bias; P.act = act; P.y = y; P.z = z;
    P.y_f32 = y_dtype == SD_F32;
    P.M = M; P.N = N; P.Kb = 2 * K;
    hipStream_t s = static_cast<hipStream_t>(stream);
    // Few rows: straight from the weights where that is one workgroup a CU (us, these kernels / tiles: 16 x 5120 x 1280 10.0 / 10.0, 64 x 1280 x 5120 22.6 / 29.5, 32 x 4096 x 4096 20.1 / 22.5, but 128 x 1280 x 1280 9.7 / 7.5)
    const int64_t r16 = (M + 15) / 16, r32 = (M + 31) / 32, c16 = (N + 15) / 16, c32 = (N + 31) / 32;
    if (r16 * c16 <= 256) return launch_few<false, true, 1, 1, 3>(P, s);
    if (r32 * c16 <= 256) return launch_few<false, true, 2, 1, 3>(P, s);
    if (M <= 32 && c32 <= 256) return launch_few<false, true, 2, 2, 2>(P, s);
    float us;
    switch (cols_choose(GATED16, M, 2ll * N, P.Kb, us)) {
    case 0: return launch_cols<COLS_BF16, 256, 256, 2, 4, 2, true, false>(P, s);
    case 1: return launch_cols<COLS_BF16, 128, 256, 2, 4, 3, true, false>(P, s);
    case 2: return launch_cols<COLS_BF16, 256, 128, 4, 2, 3, true, false>(P, s);
    case 3: return launch_cols<COLS_BF16, 128, 128, 2, 2, 3, true, false, 2>(P, s);
    case 4: return launch_cols<COLS_BF16, 64, 128, 2, 2, 3, true, false>(P, s);
    default: return launch_cols<COLS_BF16, 64, 64, 2, 1, 4, true, false, 2>(P, s);
    }
}
