// Root-mean-square norm with the residual's addition, forward and backward, for rows of 4 to 16384 elements, and rows in 8 bits, out of the norm or by themselves.
//
//   h = x + residual,  rstd = 1 / sqrt(sum_c h^2 / C + eps),  y = h rstd gamma
//   n = h rstd, g = dy gamma:  dh = rstd (g - n sum_c (g n) / C) + dres,  dgamma = sum_m dy n;  dh is the gradient of x and of the residual
//
// Bound by HBM: every element is read once and written once.  Rows lie in registers as layer norm's do (norm_rows.hpp), and the norm is of h as it is in fp32, before it is rounded
// to its type.  A block of 128 elements lies in 32 neighbouring lanes (or in 16, twice), so a row in 8 bits takes no pass of its own and no LDS.
//
// Measured (kernels alone, cold; mean and least): 8192 x 1280 bf16 onto fp32, h and 8 bits out, 18.7 and 16.8 us (115 MB, 6.1 to 6.8 TB/s); backward fp32 with the stream's gradient and the weight's 28.3 and
// 26.0 (147 MB) and 4.1 for the sums (in bf16 25.8 in the mean, 16.2 without the stream's gradient: each chunk of it is widened in a branch of its own, which waits for all loads before it asks for the next; gamma's
// chunks likewise, ahead of the first row); 10240 x 1280 bf16 quantized 9.5 and 9.0 (39 MB); one row 3.5 and 2.3.  (Of the twelve backward kernels beyond C = 4096 with the weight's gradient six keep 12 to 40
// bytes a lane in scratch.)
#include "norm_rows.hpp"
#include "fp8.hpp"

#include <algorithm>

namespace sd {

struct Fp8Out {};      // y in 8 bits
struct NoRes {};       // no residual
template <class T> struct Raw { using type = f32x4u; };
template <> struct Raw<__bf16> { using type = bf16x4u; };
template <class T> struct Bytes { using type = T; };
template <> struct Bytes<Fp8Out> { using type = uint8_t; };
template <> struct Bytes<NoRes> { using type = float; };
template <class V>
__device__ __forceinline__ f32x4 widen4(V v) { return f32x4{(float)v[0], (float)v[1], (float)v[2], (float)v[3]}; }

// As ln_fwd_kernel: a wavefront (or workgroup, or a quarter of a wavefront) takes every `stride`-th row, and asks for the next one before it works on one.
template <class X, class R, class Y, int TPR, int J, int JW>
__global__ __launch_bounds__(ln_block<TPR>()) void rms_fwd_kernel(const X* x, const typename Bytes<R>::type* res, const uint16_t* __restrict__ gamma, float eps, typename Bytes<Y>::type* y,
                                                                  uint8_t* __restrict__ scales, int64_t lds, typename Bytes<R>::type* h, float* __restrict__ rstd, int M, int C) {
    constexpr bool RES = !std::is_same_v<R, NoRes>, FP8 = std::is_same_v<Y, Fp8Out>;
    constexpr int RPB = ln_block<TPR>() / TPR;
    using XV = typename Raw<X>::type;
    using RV = typename Raw<R>::type;
    __shared__ float sh[TPR > 64 ? 32 : 1];
    const int t = threadIdx.x % TPR;
    int64_t row = (int64_t)blockIdx.x * RPB + threadIdx.x / TPR;
    const int64_t stride = (int64_t)gridDim.x * RPB;
    if (row >= M) return;        // (and in the loop: who shares a row, or an exchange between lanes, leaves together)
    const __bf16* const gb = reinterpret_cast<const __bf16*>(gamma);
    XV nx[J];
    RV nr[RES ? J : 1];
    f32x4 v[J], g[J];
    auto fetch = [&](int64_t r) {
        each_chunk<TPR, J, JW>(t, C, [&](int j, auto c) {
            nx[j] = *reinterpret_cast<const XV*>(x + r * C + c.at);
            if constexpr (RES) nr[j] = *reinterpret_cast<const RV*>(res + r * C + c.at);
        });
    };
    fetch(row);
    each_chunk<TPR, J, JW>(t, C, [&](int j, auto c) { g[j] = gamma ? load4(gb + c.at) : f32x4{1.f, 1.f, 1.f, 1.f}; });
    const float inv = 1.0f / (float)C;
    for (; row < M; row += stride) {
#pragma unroll
        for (int j = 0; j < J; ++j) {
            v[j] = widen4(nx[j]);
            if constexpr (RES) v[j] += widen4(nr[j]);
        }
        if (row + stride < M) fetch(row + stride);
        float s[1] = {0.f};
        each_chunk<TPR, J, JW>(t, C, [&](int j, auto c) {
#pragma unroll
            for (int e = 0; e < 4; ++e) s[0] += c.on(e) ? v[j][e] * v[j][e] : 0.f;
        });
        row_sums<TPR>(s, sh);
        const float r = 1.0f / sqrtf(s[0] * inv + eps);
        if (rstd && t == 0) rstd[row] = r;
        // (behind the sum's barrier: in place of the residual, and of a length that four do not divide, another thread has read what this one overwrites)
        if constexpr (RES)
            if (h) each_chunk<TPR, J, JW>(t, C, [&](int j, auto c) { c.store(h + row * C, C, v[j]); });
#pragma unroll
        for (int j = 0; j < J; ++j) v[j] = v[j] * r * g[j];
        if constexpr (!FP8) {
            each_chunk<TPR, J, JW>(t, C, [&](int j, auto c) { c.store(y + row * C, C, v[j]); });
        } else {
            // (C is a multiple of 16: a chunk is whole or not there)
            uint32_t m[J];
            each_chunk<TPR, J, JW>(t, C, [&](int j, auto c) {
                m[j] = c.on(0) ? fp8_magnitude(0, v[j]) : 0u;
                m[j] = TPR == 16 ? max16(m[j]) : max32(m[j]);
            });
            if constexpr (TPR == 16)
#pragma unroll
                for (int j = 0; j + 1 < J; j += 2) m[j] = m[j + 1] = max(m[j], m[j + 1]);
            each_chunk<TPR, J, JW>(t, C, [&](int j, auto c) {
                if (!c.on(0)) return;
                const int sc = fp8_scale(m[j]), ch = t + j * TPR;
                *reinterpret_cast<uint32_t*>(y + row * C + c.at) = fp8_pack(v[j], fp8_inverse(sc));
                if (ch % (FP8_BLOCK / 4) == 0) scales[ch / (FP8_BLOCK / 4) * lds + row] = (uint8_t)sc;
            });
        }
    }
}

// Backward, rows: as ln_bwd_rows
template <class X, class D, int TPR, int J, int JW, bool GRADS, int NT>
__device__ __forceinline__ void rms_bwd_rows(const D* dy, const X* h, const float* __restrict__ rstd, const uint16_t* __restrict__ gamma, const X* dres, X* dh, float* __restrict__ partials,
                                             int M, int C, int group, int groups) {
    constexpr int RPB = NT / TPR;
    __shared__ float sh[TPR > 64 ? 32 : 1];
    constexpr int SETS = TPR < 64 ? NT / 64 : RPB;          // sums of a column that meet in LDS
    __shared__ f32x4 comb[GRADS ? SETS * J * TPR : 1];
    const int t = threadIdx.x % TPR, sub = threadIdx.x / TPR;
    const __bf16* const gb = reinterpret_cast<const __bf16*>(gamma);
    f32x4 g[J], ag[GRADS ? J : 1];
    each_chunk<TPR, J, JW>(t, C, [&](int j, auto c) {
        g[j] = gamma ? load4(gb + c.at) : f32x4{1.f, 1.f, 1.f, 1.f};
        if (GRADS) ag[GRADS ? j : 0] = f32x4{0.f, 0.f, 0.f, 0.f};
    });
    const float inv = 1.0f / (float)C;
    for (int64_t row0 = (int64_t)group * RPB; row0 < M; row0 += (int64_t)groups * RPB) {
        // (a row past the end works on the last one, and neither adds nor stores: rows of several wavefronts meet at barriers)
        const int64_t row = min(row0 + sub, (int64_t)M - 1);
        const bool mine = row0 + sub < M;
        if (TPR <= 64 && !mine) break;
        f32x4 v[J], d[J], a[J];
        each_chunk<TPR, J, JW>(t, C, [&](int j, auto c) {
            v[j] = load4(h + row * C + c.at);
            d[j] = load4(dy + row * C + c.at);
            a[j] = dres ? load4(dres + row * C + c.at) : f32x4{0.f, 0.f, 0.f, 0.f};
        });
        const float r = rstd[row];
        float s[1] = {0.f};
        each_chunk<TPR, J, JW>(t, C, [&](int j, auto c) {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const float dd = c.on(e) ? d[j][e] : 0.f;
                v[j][e] = c.on(e) ? v[j][e] * r : 0.f;
                if (GRADS && (TPR <= 64 || mine)) ag[GRADS ? j : 0][e] += dd * v[j][e];
                d[j][e] = dd * g[j][e];
                s[0] += d[j][e] * v[j][e];
            }
        });
        row_sums<TPR>(s, sh);
        const float c1 = s[0] * inv;
        if (TPR <= 64 || mine)
            each_chunk<TPR, J, JW>(t, C, [&](int j, auto c) {
                f32x4 o;
#pragma unroll
                for (int e = 0; e < 4; ++e) o[e] = r * (d[j][e] - v[j][e] * c1) + a[j][e];
                c.store(dh + row * C, C, o);
            });
    }
    if constexpr (GRADS) {
        // the wavefronts' sums meet in LDS at once, and all threads add them up, in the order of the wavefronts
        int set = sub;
        bool lead = true;            // of the threads that hold the same columns' sums
        if constexpr (TPR < 64) {
#pragma unroll
            for (int o = TPR; o < 64; o *= 2)
#pragma unroll
                for (int j = 0; j < J; ++j)
#pragma unroll
                    for (int e = 0; e < 4; ++e) ag[j][e] += __shfl_xor(ag[j][e], o);
            set = threadIdx.x >> 6;
            lead = (threadIdx.x & 63) < TPR;
        }
        if (lead)
#pragma unroll
            for (int j = 0; j < J; ++j) comb[(set * J + j) * TPR + t] = ag[j];
        __syncthreads();
        for (int p = threadIdx.x; p < J * TPR; p += NT) {
            f32x4 v = comb[p];
#pragma unroll
            for (int w = 1; w < SETS; ++w) v += comb[w * J * TPR + p];
            Chunk<false>(p, C).store(partials + (int64_t)group * C, C, v);
        }
    }
}
// ... and 16 columns' gradients from all rows: as ln_bwd_columns
template <class X, class D, int NT>
__device__ __forceinline__ void rms_bwd_columns(const D* dy, const X* h, const float* __restrict__ rstd, float* dgamma, int M, int C, int block, int blocks) {
    constexpr int SUB = NT / 4, BATCH = 4;
    __shared__ f32x4 sh[NT / 64][4];
    const int per = (blocks + 7) / 8, mine = (block & 7) * per + (block >> 3);
    const Chunk<false> c(mine * 4 + (threadIdx.x & 3), C);
    f32x4 a = {0.f, 0.f, 0.f, 0.f};
    if ((block >> 3) < per && c.first < C)
        for (int r = threadIdx.x >> 2; r < M; r += SUB * BATCH) {
            f32x4 v[BATCH], d[BATCH];
            float s[BATCH];
#pragma unroll
            for (int i = 0; i < BATCH; ++i) {
                const int64_t row = min(r + i * SUB, M - 1);
                v[i] = load4(h + row * C + c.at);
                d[i] = load4(dy + row * C + c.at);
                s[i] = rstd[row];
            }
#pragma unroll
            for (int i = 0; i < BATCH; ++i)
                if (r + i * SUB < M)
#pragma unroll
                    for (int e = 0; e < 4; ++e) a[e] += d[i][e] * (v[i][e] * s[i]);
        }
#pragma unroll
    for (int o = 4; o < 64; o *= 2)
#pragma unroll
        for (int e = 0; e < 4; ++e) a[e] += __shfl_xor(a[e], o);
    if ((threadIdx.x & 63) < 4) sh[threadIdx.x >> 6][threadIdx.x & 3] = a;
    __syncthreads();
    if (threadIdx.x >= 4 || (block >> 3) >= per || c.first >= C) return;
    for (int w = 1; w < NT / 64; ++w) a += sh[w][threadIdx.x];
    c.store(dgamma, C, a);
}
template <class X, class D, int TPR, int J, int JW, bool GRADS, int NT>
__global__ __launch_bounds__(NT) void rms_bwd_kernel(const D* dy, const X* h, const float* __restrict__ rstd, const uint16_t* __restrict__ gamma, const X* dres, X* dh, float* __restrict__ partials, int M, int C) {
    rms_bwd_rows<X, D, TPR, J, JW, GRADS, NT>(dy, h, rstd, gamma, dres, dh, partials, M, C, blockIdx.x, gridDim.x);
}
// Few rows: both in one launch
template <class X, class D, int TPR, int J, int JW, int NT>
__global__ __launch_bounds__(NT) void rms_bwd_few_kernel(const D* dy, const X* h, const float* __restrict__ rstd, const uint16_t* __restrict__ gamma, const X* dres, X* dh, float* dgamma, int M, int C, int groups) {
    if ((int)blockIdx.x < groups) rms_bwd_rows<X, D, TPR, J, JW, false, NT>(dy, h, rstd, gamma, dres, dh, nullptr, M, C, blockIdx.x, groups);
    else rms_bwd_columns<X, D, NT>(dy, h, rstd, dgamma, M, C, (int)blockIdx.x - groups, (int)gridDim.x - groups);
}

// Rows of x in 8 bits.  16 lanes have a block, eight elements each; a wavefront U neighbouring blocks of four rows, whose loads are all in flight, a workgroup 16 rows, whose scales
// are next to each other.
template <class X, int U>
__global__ __launch_bounds__(256) void quantize_kernel(const X* __restrict__ x, uint8_t* __restrict__ q, uint8_t* __restrict__ scales, int64_t lds, int M, int K) {
    const int64_t row = (int64_t)blockIdx.x * 16 + (threadIdx.x >> 4);
    if (row >= M) return;       // (16 lanes together, and no exchange reaches beyond them)
    const int l = threadIdx.x & 15, b0 = blockIdx.y * U, blocks = (K + FP8_BLOCK - 1) / FP8_BLOCK;
    f32x8 v[U];
#pragma unroll
    for (int i = 0; i < U; ++i) {
        const int k = (b0 + i) * FP8_BLOCK + l * 8;      // (K is a multiple of 16: eight are there or not)
        v[i] = f32x8{{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
        if (k < K) v[i] = load8(x + row * K + k);
    }
#pragma unroll
    for (int i = 0; i < U; ++i) {
        if (b0 + i >= blocks) break;
        const int k = (b0 + i) * FP8_BLOCK + l * 8;
        const int sc = fp8_scale(max16(fp8_magnitude(fp8_magnitude(0, v[i].lo), v[i].hi)));
        const float inv = fp8_inverse(sc);
        if (k < K) *reinterpret_cast<u32x2*>(q + row * K + k) = u32x2{fp8_pack(v[i].lo, inv), fp8_pack(v[i].hi, inv)};
        if (l == 0) scales[(int64_t)(b0 + i) * lds + row] = (uint8_t)sc;
    }
}

constexpr int RMS_MIN_C = 4, RMS_MAX_C = 16384, FP8_MAX_M = 1 << 27, FP8_MAX_K = 1 << 22;
static int rms_check(const char* who, int x_dtype, int M, int C) {
    SD_REQUIRE(M >= 0 && C > 0, SD_EINVAL, "%s: M=%d C=%d", who, M, C);
    SD_REQUIRE(C >= RMS_MIN_C && C <= RMS_MAX_C, SD_EUNSUPPORTED, "%s: rows of %d elements (%d to %d)", who, C, RMS_MIN_C, RMS_MAX_C);
    SD_REQUIRE(x_dtype == SD_BF16 || x_dtype == SD_F32, SD_EINVAL, "%s: type %d", who, x_dtype);
    return SD_OK;
}
int fp8_check(const char* who, const char* what, const void* q, const uint8_t* scales, int64_t lds, int64_t rows, int K) {
    SD_REQUIRE(K > 0 && K % 16 == 0 && K < FP8_MAX_K, SD_EUNSUPPORTED, "%s: %s rows of %d elements in 8 bits (a multiple of 16 below 2^22)", who, what, K);
    SD_REQUIRE(q && scales, SD_EINVAL, "%s: %s: values or scales are null", who, what);
    SD_REQUIRE(aligned16(q) && aligned16(scales), SD_EINVAL, "%s: %s: pointers must be 16-byte aligned", who, what);
    SD_REQUIRE(lds >= rows && lds % 4 == 0, SD_EINVAL, "%s: %s: %lld scales between blocks (a multiple of 4, at least %lld)", who, what, (long long)lds, (long long)rows);
    return SD_OK;
}
int launch_quantize(const void* x, bool f32, uint8_t* q, uint8_t* scales, int64_t lds, int M, int K, hipStream_t stream) {
    if (SD_DRY_RUN("quantize; ")) return SD_OK;
    const int blocks = fp8_blocks(K);
    // four blocks a wavefront where that leaves four workgroups a CU
    const bool wide = (int64_t)((M + 15) / 16) * ((blocks + 3) / 4) >= 1024;
    const dim3 grid((M + 15) / 16, wide ? (blocks + 3) / 4 : blocks);
    by_type(f32 ? SD_F32 : SD_BF16, [&](auto* xt) {
        using X = std::remove_pointer_t<decltype(xt)>;
        const X* const xp = static_cast<const X*>(x);
        if (wide) hipLaunchKernelGGL((quantize_kernel<X, 4>), grid, dim3(256), 0, stream, xp, q, scales, lds, M, K);
        else hipLaunchKernelGGL((quantize_kernel<X, 1>), grid, dim3(256), 0, stream, xp, q, scales, lds, M, K);
        return 0;
    });
    SD_HIP_CHECK(hipGetLastError());
    return SD_OK;
}

static int rms_fwd_groups(int M, int C) {
    const int tpr = ln_threads_per_row(C, false), rpb = tpr > LN_THREADS ? 1 : LN_THREADS / tpr;
    return std::min((M - 1) / rpb + 1, 1024);
}
static int rms_bwd_groups(int M, int C, bool grads) {
    const int tpr = ln_threads_per_row(C, true), rpb = tpr > 512 ? 1 : 512 / tpr;
    const int groups = M > 0 ? (M - 1) / rpb + 1 : 0;
    if (!grads) return std::min(groups, C <= 768 ? 1024 : 512);
    return std::min(tpr > 64 ? (groups + 3) / 4 : groups, C <= 768 ? 512 : 256);
}
static bool rms_bwd_few(int M, int C) { return M <= 1536 && (int64_t)M * C <= 1 << 22; }

}  // namespace sd

using namespace sd;

extern "C" int sd_quantize_fp8(const void* x, int32_t x_dtype, uint8_t* q, uint8_t* scales, int64_t lds, int32_t M, int32_t K, void* stream) {
    SD_REQUIRE(M >= 0, SD_EINVAL, "quantize_fp8: M=%d", M);
    SD_REQUIRE(x_dtype == SD_BF16 || x_dtype == SD_F32, SD_EINVAL, "quantize_fp8: type %d", x_dtype);
    SD_REQUIRE(M < FP8_MAX_M, SD_EUNSUPPORTED, "quantize_fp8: M=%d (below 2^27)", M);
    SD_REQUIRE(K > 0 && K % 16 == 0 && K < FP8_MAX_K, SD_EUNSUPPORTED, "quantize_fp8: rows of %d elements (a multiple of 16 below 2^22)", K);
    if (M == 0) return SD_OK;
    const int rc = fp8_check("quantize_fp8", "result", q, scales, lds, M, K);
    if (rc) return rc;
    SD_REQUIRE(x && aligned16(x), SD_EINVAL, "quantize_fp8: x is null or not 16-byte aligned");
    SD_REQUIRE(static_cast<const void*>(q) != x && static_cast<const void*>(scales) != x && q != scales, SD_EINVAL, "quantize_fp8: a result in another's place");
    return launch_quantize(x, x_dtype == SD_F32, q, scales, lds, M, K, static_cast<hipStream_t>(stream));
}

extern "C" int sd_rmsnorm_fwd(const void* x, int32_t x_dtype, const void* residual, int32_t res_dtype, const uint16_t* gamma, float eps, void* y, int32_t y_dtype, uint8_t* scales, int64_t lds,
                              void* h, float* rstd, int32_t M, int32_t C, void* stream) {
    int rc = rms_check("rmsnorm_fwd", x_dtype, M, C);
    if (rc) return rc;
    SD_REQUIRE(y_dtype == SD_BF16 || y_dtype == SD_F32 || y_dtype == SD_FP8, SD_EINVAL, "rmsnorm_fwd: y_dtype=%d", y_dtype);
    SD_REQUIRE(!residual || res_dtype == SD_BF16 || res_dtype == SD_F32, SD_EINVAL, "rmsnorm_fwd: res_dtype=%d", res_dtype);
    SD_REQUIRE(!residual || res_dtype == SD_F32 || x_dtype == SD_BF16, SD_EUNSUPPORTED, "rmsnorm_fwd: an fp32 x onto a bf16 residual");
    SD_REQUIRE(residual || !h, SD_EINVAL, "rmsnorm_fwd: h without a residual");
    SD_REQUIRE(y_dtype != SD_FP8 || C % 16 == 0, SD_EUNSUPPORTED, "rmsnorm_fwd: rows of %d elements in 8 bits (a multiple of 16)", C);
    if (M == 0) return SD_OK;
    SD_REQUIRE(x && y, SD_EINVAL, "rmsnorm_fwd: x or y is null");
    SD_REQUIRE(aligned16(x) && aligned16(residual) && aligned16(gamma) && aligned16(y) && aligned16(h) && aligned16(rstd), SD_EINVAL, "rmsnorm_fwd: pointers must be 16-byte aligned");
    if (y_dtype == SD_FP8) {
        rc = fp8_check("rmsnorm_fwd", "y", y, scales, lds, M, C);
        if (rc) return rc;
    }
    SD_REQUIRE((y != x || y_dtype == x_dtype) && (y != residual || y_dtype == res_dtype), SD_EINVAL, "rmsnorm_fwd: in place with two types");
    SD_REQUIRE(!h || (h != y && (h != x || x_dtype == res_dtype)), SD_EINVAL, "rmsnorm_fwd: h in another's place");
    const void* const sc = y_dtype == SD_FP8 ? scales : nullptr;
    const void *const given[] = {gamma, x, residual, y, h}, *const made[] = {y, h, sc, rstd};
    for (int i = 0; i < 4; ++i)        // (y and h: as above; nothing is in gamma's place, nor a scale or a statistic in any)
        for (int j = 0; j < (i < 2 ? 1 : 5); ++j) SD_REQUIRE(!made[i] || made[i] != given[j], SD_EINVAL, "rmsnorm_fwd: a result in another's place");
    SD_REQUIRE(!sc || sc != rstd, SD_EINVAL, "rmsnorm_fwd: a result in another's place");
    if (SD_DRY_RUN("rmsnorm fwd%s; ", y_dtype == SD_FP8 ? " 8 bits" : "")) return SD_OK;
    hipStream_t s = static_cast<hipStream_t>(stream);
    auto run = [&](auto xt, auto rt, auto yt) {
        using X = decltype(xt);
        using R = decltype(rt);
        using Y = decltype(yt);
        using RT = typename Bytes<R>::type;
        return ln_by_length<false>(C, [&](auto shape) {
            using S = decltype(shape);
            hipLaunchKernelGGL((rms_fwd_kernel<X, R, Y, S::TPR, S::J, S::JW>), dim3(rms_fwd_groups(M, C)), dim3(ln_block<S::TPR>()), 0, s, static_cast<const X*>(x), static_cast<const RT*>(residual), gamma,
                               eps, static_cast<typename Bytes<Y>::type*>(y), scales, lds, static_cast<RT*>(h), rstd, M, C);
            SD_HIP_CHECK(hipGetLastError());
            return (int)SD_OK;
        });
    };
    auto by_y = [&](auto xt, auto rt) {
        if (y_dtype == SD_FP8) return run(xt, rt, Fp8Out());
        if (y_dtype == SD_F32) return run(xt, rt, 0.f);
        return run(xt, rt, __bf16());
    };
    if (x_dtype == SD_F32) return residual ? by_y(0.f, 0.f) : by_y(0.f, NoRes());
    if (!residual) return by_y(__bf16(), NoRes());
    return res_dtype == SD_F32 ? by_y(__bf16(), 0.f) : by_y(__bf16(), __bf16());
}

extern "C" size_t sd_rmsnorm_bwd_workspace_bytes(int32_t M, int32_t C) {
    if (M <= 0 || C <= 0) return 256;
    return round_up((size_t)rms_bwd_groups(M, C, true) * C * 4, 256);
}

extern "C" int sd_rmsnorm_bwd(const void* dy, int32_t y_dtype, const void* h, int32_t h_dtype, const float* rstd, const uint16_t* gamma, const void* dres, void* dh, float* dgamma, int32_t M, int32_t C,
                              void* ws, size_t ws_bytes, void* stream) {
    int rc = rms_check("rmsnorm_bwd", h_dtype, M, C);
    if (rc) return rc;
    SD_REQUIRE(y_dtype == SD_BF16 || y_dtype == SD_F32, SD_EINVAL, "rmsnorm_bwd: y_dtype=%d", y_dtype);
    SD_REQUIRE(M == 0 || (dy && h && rstd && dh), SD_EINVAL, "rmsnorm_bwd: dy, h, rstd or dh is null");
    SD_REQUIRE(aligned16(dy) && aligned16(h) && aligned16(rstd) && aligned16(gamma) && aligned16(dres) && aligned16(dh) && aligned16(dgamma), SD_EINVAL, "rmsnorm_bwd: pointers must be 16-byte aligned");
    SD_REQUIRE(M == 0 || dh != dy || h_dtype == y_dtype, SD_EINVAL, "rmsnorm_bwd: in place of dy with two types");
    SD_REQUIRE(M == 0 || (dh != rstd && dh != gamma && dh != dgamma), SD_EINVAL, "rmsnorm_bwd: dh in another's place");
    for (const void* in : {dy, h, dres, static_cast<const void*>(rstd), static_cast<const void*>(gamma)})
        SD_REQUIRE(M == 0 || !dgamma || dgamma != in, SD_EINVAL, "rmsnorm_bwd: dgamma in an input's place");
    hipStream_t s = static_cast<hipStream_t>(stream);
    if (M == 0) return dgamma ? launch_sum_partials(nullptr, 0, dgamma, C, nullptr, 0, s) : SD_OK;    // sums over no rows
    // (not in place: a row may be overwritten before a column has read it)
    const bool few = dgamma && rms_bwd_few(M, C) && dh != h && dh != dy;
    float* partials = nullptr;
    if (dgamma) {
        Workspace w(ws, ws_bytes);
        const size_t need = sd_rmsnorm_bwd_workspace_bytes(M, C);
        partials = static_cast<float*>(w.take(need));
        SD_REQUIRE(partials && w.ok() && (reinterpret_cast<uintptr_t>(ws) & 255u) == 0, SD_EWORKSPACE, "rmsnorm_bwd: workspace of %zu bytes, need %zu, 256-byte aligned", ws_bytes, need);
    }
    const int groups = rms_bwd_groups(M, C, dgamma && !few);
    if (!SD_DRY_RUN("rmsnorm bwd%s; ", few ? " few" : "")) {
        rc = by_type(h_dtype, [&](auto* xt) {
            return by_type(y_dtype, [&](auto* yt) {
                return ln_by_length<true>(C, [&](auto shape) {
                    using X = std::remove_pointer_t<decltype(xt)>;
                    using D = std::remove_pointer_t<decltype(yt)>;
                    using S = decltype(shape);
                    constexpr int NT = ln_bwd_threads(S::TPR);
                    const D* const d = static_cast<const D*>(dy);
                    const X *const hp = static_cast<const X*>(h), *const rp = static_cast<const X*>(dres);
                    X* const o = static_cast<X*>(dh);
                    if (few)
                        hipLaunchKernelGGL((rms_bwd_few_kernel<X, D, S::TPR, S::J, S::JW, NT>), dim3(groups + ((C + 15) / 16 + 7) / 8 * 8), dim3(NT), 0, s, d, hp, rstd, gamma, rp, o, dgamma, M, C, groups);
                    else if (dgamma)
                        hipLaunchKernelGGL((rms_bwd_kernel<X, D, S::TPR, S::J, S::JW, true, NT>), dim3(groups), dim3(NT), 0, s, d, hp, rstd, gamma, rp, o, partials, M, C);
                    else
                        hipLaunchKernelGGL((rms_bwd_kernel<X, D, S::TPR, S::J, S::JW, false, NT>), dim3(groups), dim3(NT), 0, s, d, hp, rstd, gamma, rp, o, partials, M, C);
                    SD_HIP_CHECK(hipGetLastError());
                    return (int)SD_OK;
                });
            });
        });
        if (rc) return rc;
    }
    return dgamma && !few ? launch_sum_partials(partials, groups, dgamma, C, nullptr, 0, s) : SD_OK;
}
