// A gated linear layer in bf16, as in training:
//
//   v = x Wv^T + bv,  g = x Wg^T + bg,  y = v act(g),  W = [Wv; Wg]
//
// Both projections, the activation and the product in one kernel (gemm_cols.hpp); v and g are kept in bf16 where the backward pass (linear.hip) wants them.
#include "gemm_cols.hpp"

#include <string.h>

using namespace sd;

extern "C" int sd_gated_linear_fwd(const uint16_t* x, const uint16_t* W, const uint16_t* bias, int32_t act, void* y, int32_t y_dtype, uint16_t* z, int32_t M, int32_t N, int32_t K, void* stream) {
    SD_REQUIRE(M >= 0 && N >= 0, SD_EINVAL, "gated_linear_fwd: M=%d N=%d", M, N);
    SD_REQUIRE(K > 0 && K % 8 == 0, SD_EUNSUPPORTED, "gated_linear_fwd: K=%d is not a positive multiple of 8", K);
    SD_REQUIRE(M < (1 << 27) && N < (1 << 21) && K < (1 << 22), SD_EUNSUPPORTED, "gated_linear_fwd: M=%d N=%d K=%d (M below 2^27, N below 2^21, K below 2^22)", M, N, K);
    SD_REQUIRE(act >= SD_ACT_NONE && act <= SD_ACT_RELU, SD_EINVAL, "gated_linear_fwd: activation %d", act);
    SD_REQUIRE(y_dtype == SD_BF16 || y_dtype == SD_F32, SD_EINVAL, "gated_linear_fwd: y_dtype=%d", y_dtype);
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
    if (M <= 16) return launch_few<false, true, 1, 1, 3>(P, s);
    if (M <= 512) return launch_cols<COLS_BF16, 64, 128, 2, 2, 3, true, false>(P, s);
    return launch_cols<COLS_BF16, 256, 256, 4, 2, 2, true, false>(P, s);
}
