// Layer norm as an operator of its own, forward and backward, for rows of 4 to 16384 elements in fp32 or bf16.
// (The one in norm.hip feeds a projection of the transformer block: bf16 out, and it clears flags and reads weights ahead.)
//
//   mean = sum_c x / C,  rstd = 1 / sqrt(sum_c (x - mean)^2 / C + eps),  y = (x - mean) rstd gamma + beta
//   n = (x - mean) rstd, g = dy gamma:  dx = rstd (g - sum_c g / C - n sum_c (g n) / C),
//   dgamma = sum_m dy n,  dbeta = sum_m dy
//
// Bound by HBM: every element is read once and written once.  A row lives in the registers of TPR threads, four elements a
// chunk, and all of its loads are issued before the first is used.  Statistics are fp32 and taken in two steps over the
// registers: a mean, then the sums of the deviations and of their squares, of which the first corrects the mean's own
// rounding.  (One pass over sums and squares loses the variance's digits where a row has a large offset, or one
// element far from all others.)
//
// Measured, 8192 x 1280 fp32 to bf16 (kernels alone, three sets of inputs in turn): forward 14.2 us, 4.4 TB/s; backward with gradients of the weights 20.9 and 4.0 for the sums; 2777 x 1155
// bf16 11.5 + 3.6.  From cold inputs into cold results 17.6 (a copy of the same 63 MB: 14.0) and 27.8 in all (a copy of 105 MB 22.3).  Stores past the caches make the forward pass 16.4
// cold, and the projection behind it slower by more than that.
// Other rows, cold (forward / backward with gradients of the weights / without): 8192 x 1280 bf16 13.9 / 20.6 / 16.5, 8192 x 1155 bf16 14.1 / 21.4 / 16.4, 32768 x 320 fp32 to bf16 16.4 /
// 27.1 / 26.3; few long ones 1024 x 8192 fp32 to bf16 18.0 / 39.2 / 24.7, 1024 x 16384 34.4 / 60.2 / 39.0 (of the eight backward kernels beyond C = 4096 with gradients of the weights four
// keep 4 to 14 registers in scratch).
#include "rows.hpp"

#include <algorithm>

namespace sd {

// sums over the TPR threads of a row, in every one of them
template <int TPR, int N>
__device__ __forceinline__ void row_sums(float (&v)[N], float* sh) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
        if constexpr (TPR == 16) v[i] = dpp_add(dpp_add(dpp_add(dpp_add(v[i], 0), 1), 2), 3);
        else v[i] = wave_sum(v[i]);
    }
    if constexpr (TPR > 64) {
        constexpr int W = TPR / 64;
        const int first = threadIdx.x / TPR * W, wave = threadIdx.x >> 6;      // (of this row's wavefronts)
        __syncthreads();                   // the last sums have been read
        if ((threadIdx.x & 63) == 0)
#pragma unroll
            for (int i = 0; i < N; ++i) sh[i * 16 + wave] = v[i];
        __syncthreads();
#pragma unroll
        for (int i = 0; i < N; ++i) {
            v[i] = 0.f;
#pragma unroll
            for (int w = 0; w < W; ++w) v[i] += sh[i * 16 + first + w];
        }
    }
}

// Chunk j of thread t holds elements [at, at + 4), at = 4 (t + j TPR); the last chunk of a row whose length is no multiple
// of four begins earlier, at C - 4, and the elements that its neighbour has too are off there, as are all of those
// behind the row's end.  WHOLE: a chunk that every row of this kernel has whole.
template <bool WHOLE>
struct Chunk {
    int at, first;      // where it begins; its first element that counts (C: none does)
    __device__ __forceinline__ Chunk(int ch, int C) {
        first = WHOLE ? 4 * ch : min(4 * ch, C);
        at = WHOLE ? 4 * ch : min(4 * ch, C - 4);
    }
    __device__ __forceinline__ bool on(int e) const { return WHOLE || at + e >= first; }
    template <class T>
    __device__ __forceinline__ void store(T* p, int C, f32x4 v) const {
        if (WHOLE || at == first) store4(p + at, v);
        else if (first < C)
#pragma unroll
            for (int e = 1; e < 4; ++e)
                if (on(e)) p[at + e] = (T)v[e];
    }
};
// f(j, chunk) for the J chunks of thread t, of which the first JW are whole
template <int TPR, int J, int JW, class F>
__device__ __forceinline__ void each_chunk(int t, int C, F f) {
#pragma unroll
    for (int j = 0; j < JW; ++j) f(j, Chunk<true>(t + j * TPR, C));
#pragma unroll
    for (int j = JW; j < J; ++j) f(j, Chunk<false>(t + j * TPR, C));
}

constexpr int LN_THREADS = 256;
constexpr int ln_bwd_threads(int tpr) { return tpr > 512 ? tpr : 512; }
template <int TPR>
constexpr int ln_block() { return TPR > LN_THREADS ? TPR : LN_THREADS; }

// A wavefront (or workgroup) takes every `gridDim.x`-th row of its kind, and asks for the next one before it works on one: gamma and beta are
// read once, and the loads of a row fly while the one before is reduced and stored.
template <class X, class Y, int TPR, int J, int JW>
__global__ __launch_bounds__(ln_block<TPR>()) void ln_fwd_kernel(const X* x, const uint16_t* __restrict__ gamma, const uint16_t* __restrict__ beta,
                                                                 float eps, Y* y, float* __restrict__ mean, float* __restrict__ rstd, int M, int C) {
    constexpr int RPB = ln_block<TPR>() / TPR;
    __shared__ float sh[TPR > 64 ? 32 : 1];
    const int t = threadIdx.x % TPR;
    int64_t row = (int64_t)blockIdx.x * RPB + threadIdx.x / TPR;
    const int64_t stride = (int64_t)gridDim.x * RPB;
    // Rows leave here and in the loop below at times of their own.  Of 256 threads and more a row, the workgroup is the row, and its barriers are met by all; of 64 a wavefront leaves; of
    // 16 a quarter of one, and row_sums reads no lane outside it (a wider exchange would read lanes that have left).
    if (row >= M) return;
    const __bf16* const gb = reinterpret_cast<const __bf16*>(gamma);
    const __bf16* const bb = reinterpret_cast<const __bf16*>(beta);
    f32x4 next[J], v[J], g[J], b[J];
    each_chunk<TPR, J, JW>(t, C, [&](int j, auto c) { next[j] = load4(x + row * C + c.at); });
    each_chunk<TPR, J, JW>(t, C, [&](int j, auto c) {
        g[j] = gamma ? load4(gb + c.at) : f32x4{1.f, 1.f, 1.f, 1.f};
        b[j] = beta ? load4(bb + c.at) : f32x4{0.f, 0.f, 0.f, 0.f};
    });
    const float inv = 1.0f / (float)C;
    for (; row < M; row += stride) {
#pragma unroll
        for (int j = 0; j < J; ++j) v[j] = next[j];
        if (row + stride < M) each_chunk<TPR, J, JW>(t, C, [&](int j, auto c) { next[j] = load4(x + (row + stride) * C + c.at); });
        float s[2] = {0.f, 0.f}, one[1] = {0.f};
        each_chunk<TPR, J, JW>(t, C, [&](int j, auto c) {
#pragma unroll
            for (int e = 0; e < 4; ++e) one[0] += c.on(e) ? v[j][e] : 0.f;
        });
        row_sums<TPR>(one, sh);
        const float m0 = one[0] * inv;
        each_chunk<TPR, J, JW>(t, C, [&](int j, auto c) {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                v[j][e] -= m0;
                const float d = c.on(e) ? v[j][e] : 0.f;
                s[0] += d;
                s[1] += d * d;
            }
        });
        row_sums<TPR>(s, sh);
        const float dm = s[0] * inv;
        float var = s[1] * inv - dm * dm;
        var = var < 0.f ? 0.f : var;       // (NaN stays)
        const float r = 1.0f / sqrtf(var + eps);
        if (mean && t == 0) mean[row] = m0 + dm;
        if (rstd && t == 0) rstd[row] = r;
        Y* const yr = y + row * C;
        each_chunk<TPR, J, JW>(t, C, [&](int j, auto c) {
            f32x4 o;
#pragma unroll
            for (int e = 0; e < 4; ++e) o[e] = (v[j][e] - dm) * r * g[j][e] + b[j][e];
            c.store(yr, C, o);
        });
    }
}

// Backward, rows: a workgroup takes every `groups`-th group of rows.  GRADS: it keeps the sums of its columns in registers and leaves them in
// partials[group], gradient of gamma first, for sum_partials to add up.  (The next row's loads ahead of a row's work, as in the
// forward kernel, gain nothing here: a row is two rows of loads, and the registers cost wavefronts; 8192 x 1280 bf16 17.8 us against 16.4.)
template <class X, class D, int TPR, int J, int JW, bool GRADS, int NT>
__device__ __forceinline__ void ln_bwd_rows(const D* dy, const X* x, const float* __restrict__ mean, const float* __restrict__ rstd, const uint16_t* __restrict__ gamma,
                                            X* dx, float* __restrict__ partials, int M, int C, int group, int groups) {
    constexpr int RPB = NT / TPR;
    __shared__ float sh[TPR > 64 ? 32 : 1];
    constexpr int SETS = TPR < 64 ? NT / 64 : RPB;          // sums of a column that meet in LDS
    __shared__ f32x4 comb[GRADS ? SETS * 2 * J * TPR : 1];
    const int t = threadIdx.x % TPR, sub = threadIdx.x / TPR;
    const __bf16* const gb = reinterpret_cast<const __bf16*>(gamma);
    f32x4 g[J], ag[GRADS ? J : 1], ab[GRADS ? J : 1];
    each_chunk<TPR, J, JW>(t, C, [&](int j, auto c) {
        g[j] = gamma ? load4(gb + c.at) : f32x4{1.f, 1.f, 1.f, 1.f};
        if (GRADS) ag[GRADS ? j : 0] = ab[GRADS ? j : 0] = f32x4{0.f, 0.f, 0.f, 0.f};
    });
    const float inv = 1.0f / (float)C;
    for (int64_t row0 = (int64_t)group * RPB; row0 < M; row0 += (int64_t)groups * RPB) {
        // (a row past the end works on the last one, and neither adds nor stores: rows of several wavefronts meet at barriers)
        const int64_t row = min(row0 + sub, (int64_t)M - 1);
        const bool mine = row0 + sub < M;
        if (TPR <= 64 && !mine) break;
        f32x4 v[J], d[J];
        each_chunk<TPR, J, JW>(t, C, [&](int j, auto c) {
            v[j] = load4(x + row * C + c.at);
            d[j] = load4(dy + row * C + c.at);
        });
        const float m = mean[row], r = rstd[row];
        float s[2] = {0.f, 0.f};
        each_chunk<TPR, J, JW>(t, C, [&](int j, auto c) {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const float dd = c.on(e) ? d[j][e] : 0.f;
                v[j][e] = c.on(e) ? (v[j][e] - m) * r : 0.f;
                if (GRADS && (TPR <= 64 || mine)) {
                    ag[GRADS ? j : 0][e] += dd * v[j][e];
                    ab[GRADS ? j : 0][e] += dd;
                }
                d[j][e] = dd * g[j][e];
                s[0] += d[j][e];
                s[1] += d[j][e] * v[j][e];
            }
        });
        row_sums<TPR>(s, sh);
        const float c1 = s[0] * inv, c2 = s[1] * inv;
        if (TPR <= 64 || mine)
            each_chunk<TPR, J, JW>(t, C, [&](int j, auto c) {
                f32x4 o;
#pragma unroll
                for (int e = 0; e < 4; ++e) o[e] = r * (d[j][e] - c1 - v[j][e] * c2);
                c.store(dx + row * C, C, o);
            });
    }
    if constexpr (GRADS) {
        float* const out = partials + (int64_t)group * 2 * C;
        // the wavefronts' sums meet in LDS at once, and all threads add them up, in the order of the wavefronts
        int set = sub;
        bool lead = true;            // of the threads that hold the same columns' sums
        if constexpr (TPR < 64) {
#pragma unroll
            for (int o = TPR; o < 64; o *= 2)
#pragma unroll
                for (int j = 0; j < J; ++j)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        ag[j][e] += __shfl_xor(ag[j][e], o);
                        ab[j][e] += __shfl_xor(ab[j][e], o);
                    }
            set = threadIdx.x >> 6;
            lead = (threadIdx.x & 63) < TPR;
        }
        if (lead)
#pragma unroll
            for (int j = 0; j < J; ++j) {
                comb[(set * 2 * J + j) * TPR + t] = ag[j];
                comb[(set * 2 * J + J + j) * TPR + t] = ab[j];
            }
        __syncthreads();
        for (int p = threadIdx.x; p < 2 * J * TPR; p += NT) {
            f32x4 v = comb[p];
#pragma unroll
            for (int w = 1; w < SETS; ++w) v += comb[w * 2 * J * TPR + p];
            const bool beta = p >= J * TPR;
            Chunk<false>(p - (beta ? J * TPR : 0), C).store(out + (beta ? C : 0), C, v);
        }
    }
}
// ... and 16 columns' gradients from all rows, which need no row's sums: four threads a row, NT / 4 rows at a time, four of those in flight.  Neighbouring columns go to the same XCD, whose
// L2 then holds the lines that they share.
template <class X, class D, int NT>
__device__ __forceinline__ void ln_bwd_columns(const D* dy, const X* x, const float* __restrict__ mean, const float* __restrict__ rstd, float* dgamma, float* dbeta, int M, int C, int block, int blocks) {
    constexpr int SUB = NT / 4, BATCH = 4;
    __shared__ f32x4 sh[2][NT / 64][4];
    const int per = (blocks + 7) / 8, mine = (block & 7) * per + (block >> 3);
    const Chunk<false> c(mine * 4 + (threadIdx.x & 3), C);
    f32x4 a = {0.f, 0.f, 0.f, 0.f}, b = a;
    if ((block >> 3) < per && c.first < C)
        for (int r = threadIdx.x >> 2; r < M; r += SUB * BATCH) {
            f32x4 v[BATCH], d[BATCH];
            float m[BATCH], s[BATCH];
#pragma unroll
            for (int i = 0; i < BATCH; ++i) {
                const int64_t row = min(r + i * SUB, M - 1);
                v[i] = load4(x + row * C + c.at);
                d[i] = load4(dy + row * C + c.at);
                m[i] = mean[row];
                s[i] = rstd[row];
            }
#pragma unroll
            for (int i = 0; i < BATCH; ++i)
                if (r + i * SUB < M)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        a[e] += d[i][e] * ((v[i][e] - m[i]) * s[i]);
                        b[e] += d[i][e];
                    }
        }
#pragma unroll
    for (int o = 4; o < 64; o *= 2)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            a[e] += __shfl_xor(a[e], o);
            b[e] += __shfl_xor(b[e], o);
        }
    if ((threadIdx.x & 63) < 4) {
        sh[0][threadIdx.x >> 6][threadIdx.x & 3] = a;
        sh[1][threadIdx.x >> 6][threadIdx.x & 3] = b;
    }
    __syncthreads();
    if (threadIdx.x >= 4 || (block >> 3) >= per || c.first >= C) return;
    for (int w = 1; w < NT / 64; ++w) {
        a += sh[0][w][threadIdx.x];
        b += sh[1][w][threadIdx.x];
    }
    if (dgamma) c.store(dgamma, C, a);
    if (dbeta) c.store(dbeta, C, b);
}
template <class X, class D, int TPR, int J, int JW, bool GRADS, int NT>
__global__ __launch_bounds__(NT) void ln_bwd_kernel(const D* dy, const X* x, const float* __restrict__ mean, const float* __restrict__ rstd, const uint16_t* __restrict__ gamma,
                                                    X* dx, float* __restrict__ partials, int M, int C) {
    ln_bwd_rows<X, D, TPR, J, JW, GRADS, NT>(dy, x, mean, rstd, gamma, dx, partials, M, C, blockIdx.x, gridDim.x);
}
// Few rows: both in one launch.  The column workgroups read the rows a second time, out of the caches, which costs less than a launch.
template <class X, class D, int TPR, int J, int JW, int NT>
__global__ __launch_bounds__(NT) void ln_bwd_few_kernel(const D* dy, const X* x, const float* __restrict__ mean, const float* __restrict__ rstd, const uint16_t* __restrict__ gamma,
                                                        X* dx, float* dgamma, float* dbeta, int M, int C, int groups) {
    if ((int)blockIdx.x < groups) ln_bwd_rows<X, D, TPR, J, JW, false, NT>(dy, x, mean, rstd, gamma, dx, nullptr, M, C, blockIdx.x, groups);
    else ln_bwd_columns<X, D, NT>(dy, x, mean, rstd, dgamma, dbeta, M, C, (int)blockIdx.x - groups, (int)gridDim.x - groups);
}

// 16 columns a workgroup, 32 rows at a time, so that nearly all of its loads are in flight together; the sums of a column's 32 threads are added in a fixed order.
__global__ __launch_bounds__(512) void sum_partials_kernel(const float* __restrict__ partials, int G, float* __restrict__ out0, int n0, float* __restrict__ out1, int n1) {
    __shared__ float sh[8][16];
    const int n = n0 + n1, c = blockIdx.x * 16 + (threadIdx.x & 15), at = min(c, n - 1);
    float a = 0.f;
#pragma unroll 8
    for (int g = threadIdx.x >> 4; g < G; g += 32) a += partials[(int64_t)g * n + at];
    a += __shfl_xor(a, 16);
    a += __shfl_xor(a, 32);
    if ((threadIdx.x & 63) < 16) sh[threadIdx.x >> 6][threadIdx.x & 15] = a;
    __syncthreads();
    if (threadIdx.x >= 16 || c >= n) return;
#pragma unroll
    for (int w = 1; w < 8; ++w) a += sh[w][threadIdx.x];
    float* const out = c < n0 ? out0 : out1;
    if (out) out[c < n0 ? c : c - n0] = a;
}
int launch_sum_partials(const float* partials, int G, float* out0, int n0, float* out1, int n1, hipStream_t stream) {
    if (SD_DRY_RUN("sum partials; ")) return SD_OK;
    hipLaunchKernelGGL(sum_partials_kernel, dim3((n0 + n1 + 15) / 16), dim3(512), 0, stream, partials, G, out0, n0, out1, n1);
    SD_HIP_CHECK(hipGetLastError());
    return SD_OK;
}

// Threads a row and chunks a thread, from the row's length: a wavefront up to 2048 elements, 256 threads up to 8192, and 16 threads for short rows, of which a wavefront's
// lanes would have little each (us, 64 / 16 threads a row: 32768 rows forward of 64 10.7 / 4.8, of 128 11.8 / 8.2, of 320 19.3 / 14.1; backward with gradients of the weights of 64 15.3 / 9.6, of 128
// 17.0 / 14.4, but of 256 19.7 / 25.3, 320 25.8 / 27.8: a thread's sums of columns take the registers of the wavefronts that would hide its loads).
template <int TPR_, int J_, int JW_>
struct LnShape { static constexpr int TPR = TPR_, J = J_, JW = JW_; };
template <bool BACKWARD, class F>
static int ln_by_length(int C, F f) {
    if (C <= 16 * 4) return f(LnShape<16, 1, 0>());
    if (C <= 16 * 4 * 2) return f(LnShape<16, 2, 1>());
    if constexpr (BACKWARD) {
        if (C <= 64 * 4) return f(LnShape<64, 1, 0>());
    } else {
        if (C <= 16 * 4 * 5) return f(LnShape<16, 5, 2>());
        if (C <= 16 * 4 * 8) return f(LnShape<16, 8, 5>());
    }
    if (C <= 64 * 4 * 3) return f(LnShape<64, 3, 1>());
    if (C <= 64 * 4 * 5) return f(LnShape<64, 5, 3>());
    if (C <= 64 * 4 * 8) return f(LnShape<64, 8, 5>());
    if (C <= 256 * 4 * 4) return f(LnShape<256, 4, 2>());
    if (C <= 256 * 4 * 8) return f(LnShape<256, 8, 4>());
    return f(LnShape<1024, 4, 2>());
}
static int ln_threads_per_row(int C, bool backward) { return C <= (backward ? 128 : 512) ? 16 : C <= 2048 ? 64 : C <= 8192 ? 256 : 1024; }
template <class F>
static int by_type(int dtype, F f) {
    if (dtype == SD_F32) return f(static_cast<float*>(nullptr));
    return f(static_cast<__bf16*>(nullptr));
}

constexpr int LN_MIN_C = 4, LN_MAX_C = 16384;
static int ln_check(const char* who, int x_dtype, int y_dtype, int M, int C) {
    SD_REQUIRE(M >= 0 && C > 0, SD_EINVAL, "%s: M=%d C=%d", who, M, C);
    SD_REQUIRE(C >= LN_MIN_C && C <= LN_MAX_C, SD_EUNSUPPORTED, "%s: rows of %d elements (%d to %d)", who, C, LN_MIN_C, LN_MAX_C);
    SD_REQUIRE((x_dtype == SD_BF16 || x_dtype == SD_F32) && (y_dtype == SD_BF16 || y_dtype == SD_F32), SD_EINVAL, "%s: types %d, %d", who, x_dtype, y_dtype);
    return SD_OK;
}

// Workgroups of the forward pass: four a CU, or one for every group of rows where there are fewer
static int ln_fwd_groups(int M, int C) {
    const int tpr = ln_threads_per_row(C, false), rpb = tpr > LN_THREADS ? 1 : LN_THREADS / tpr;
    return std::min((M - 1) / rpb + 1, 1024);
}
// ... of the backward pass, eight wavefronts each.  With gradients of the weights one a CU, of short rows two: their sums of columns are written and read again (us at 128 / 256 /
// 512 workgroups: 8192 x 1280 fp32 31.8 / 29.9 / 33.9, 2777 x 1155 bf16 17.3 / 16.4 / 21.7, 32768 x 320 51.6 / 32.3 / 26.4), and of rows that take a workgroup no fewer than four rows to
// each (500 x 4096, 500 / 125 workgroups, 21.0 / 13.3).  Without twice as many.
static int ln_bwd_groups(int M, int C, bool grads) {
    const int tpr = ln_threads_per_row(C, true), rpb = tpr > 512 ? 1 : 512 / tpr;
    const int groups = M > 0 ? (M - 1) / rpb + 1 : 0;
    if (!grads) return std::min(groups, C <= 768 ? 1024 : 512);
    return std::min(tpr > 64 ? (groups + 3) / 4 : groups, C <= 768 ? 512 : 256);
}
// Few rows, all in one launch: what the columns read a second time lies in the caches, but there are few of their workgroups (us, two launches / one: 3 x 950 6.1 / 3.1, 300 x 1280 8.6 / 5.1, 1000 x 640 8.4 /
// 6.6, 500 x 4096 15.8 / 7.4, 1200 x 1000 10.1 / 7.2, 2048 x 1280 14.7 / 15.0, 2777 x 1155 15.2 / 16.5, 4096 x 1280 15.7 / 23.8).
static bool ln_bwd_few(int M, int C) { return M <= 1536 && (int64_t)M * C <= 1 << 22; }

}  // namespace sd

using namespace sd;

extern "C" int sd_layernorm_fwd(const void* x, int32_t x_dtype, const uint16_t* gamma, const uint16_t* beta, float eps, void* y, int32_t y_dtype,
                                float* mean, float* rstd, int32_t M, int32_t C, void* stream) {
    int rc = ln_check("layernorm_fwd", x_dtype, y_dtype, M, C);
    if (rc) return rc;
    if (M == 0) return SD_OK;
    SD_REQUIRE(x && y, SD_EINVAL, "layernorm_fwd: x or y is null");
    SD_REQUIRE(aligned16(x) && aligned16(y) && aligned16(gamma) && aligned16(beta) && aligned16(mean) && aligned16(rstd), SD_EINVAL,
               "layernorm_fwd: pointers must be 16-byte aligned");
    SD_REQUIRE(x != y || x_dtype == y_dtype, SD_EINVAL, "layernorm_fwd: in place with two types");
    if (SD_DRY_RUN("layernorm fwd; ")) return SD_OK;
    hipStream_t s = static_cast<hipStream_t>(stream);
    return by_type(x_dtype, [&](auto* xt) {
        return by_type(y_dtype, [&](auto* yt) {
            return ln_by_length<false>(C, [&](auto shape) {
                using X = std::remove_pointer_t<decltype(xt)>;
                using Y = std::remove_pointer_t<decltype(yt)>;
                using S = decltype(shape);
                constexpr int B = ln_block<S::TPR>();
                hipLaunchKernelGGL((ln_fwd_kernel<X, Y, S::TPR, S::J, S::JW>), dim3(ln_fwd_groups(M, C)), dim3(B), 0, s, static_cast<const X*>(x), gamma, beta, eps,
                                   static_cast<Y*>(y), mean, rstd, M, C);
                SD_HIP_CHECK(hipGetLastError());
                return (int)SD_OK;
            });
        });
    });
}

extern "C" size_t sd_layernorm_bwd_workspace_bytes(int32_t M, int32_t C) {
    if (M <= 0 || C <= 0) return 256;
    return round_up((size_t)ln_bwd_groups(M, C, true) * 2 * C * 4, 256);
}

extern "C" int sd_layernorm_bwd(const void* dy, int32_t y_dtype, const void* x, int32_t x_dtype, const float* mean, const float* rstd, const uint16_t* gamma,
                                void* dx, float* dgamma, float* dbeta, int32_t M, int32_t C, void* ws, size_t ws_bytes, void* stream) {
    int rc = ln_check("layernorm_bwd", x_dtype, y_dtype, M, C);
    if (rc) return rc;
    const bool grads = dgamma || dbeta;
    SD_REQUIRE(M == 0 || (dy && x && mean && rstd && dx), SD_EINVAL, "layernorm_bwd: dy, x, mean, rstd or dx is null");
    SD_REQUIRE(aligned16(dy) && aligned16(x) && aligned16(mean) && aligned16(rstd) && aligned16(gamma) && aligned16(dx) && aligned16(dgamma) && aligned16(dbeta), SD_EINVAL,
               "layernorm_bwd: pointers must be 16-byte aligned");
    SD_REQUIRE(M == 0 || dx != dy || x_dtype == y_dtype, SD_EINVAL, "layernorm_bwd: in place of dy with two types");
    hipStream_t s = static_cast<hipStream_t>(stream);
    if (M == 0) return grads ? launch_sum_partials(nullptr, 0, dgamma, C, dbeta, C, s) : SD_OK;    // sums over no rows
    // (not in place: a row may be overwritten before a column has read it)
    const bool few = grads && ln_bwd_few(M, C) && dx != x && dx != dy;
    float* partials = nullptr;
    if (grads) {
        Workspace w(ws, ws_bytes);
        const size_t need = sd_layernorm_bwd_workspace_bytes(M, C);
        partials = static_cast<float*>(w.take(need));
        SD_REQUIRE(partials && w.ok() && (reinterpret_cast<uintptr_t>(ws) & 255u) == 0, SD_EWORKSPACE, "layernorm_bwd: workspace of %zu bytes, need %zu, 256-byte aligned", ws_bytes, need);
    }
    const int groups = ln_bwd_groups(M, C, grads && !few);
    if (!SD_DRY_RUN("layernorm bwd%s; ", few ? " few" : "")) {
        rc = by_type(x_dtype, [&](auto* xt) {
            return by_type(y_dtype, [&](auto* yt) {
                return ln_by_length<true>(C, [&](auto shape) {
                    using X = std::remove_pointer_t<decltype(xt)>;
                    using D = std::remove_pointer_t<decltype(yt)>;
                    using S = decltype(shape);
                    constexpr int NT = ln_bwd_threads(S::TPR);
                    const D* const d = static_cast<const D*>(dy);
                    const X* const xp = static_cast<const X*>(x);
                    X* const o = static_cast<X*>(dx);
                    if (few)
                        hipLaunchKernelGGL((ln_bwd_few_kernel<X, D, S::TPR, S::J, S::JW, NT>), dim3(groups + ((C + 15) / 16 + 7) / 8 * 8), dim3(NT), 0, s, d, xp, mean, rstd, gamma, o, dgamma, dbeta, M, C, groups);
                    else if (grads)
                        hipLaunchKernelGGL((ln_bwd_kernel<X, D, S::TPR, S::J, S::JW, true, NT>), dim3(groups), dim3(NT), 0, s, d, xp, mean, rstd, gamma, o, partials, M, C);
                    else
                        hipLaunchKernelGGL((ln_bwd_kernel<X, D, S::TPR, S::J, S::JW, false, NT>), dim3(groups), dim3(NT), 0, s, d, xp, mean, rstd, gamma, o, partials, M, C);
                    SD_HIP_CHECK(hipGetLastError());
                    return (int)SD_OK;
                });
            });
        });
        if (rc) return rc;
    }
    return grads && !few ? launch_sum_partials(partials, groups, dgamma, C, dbeta, C, s) : SD_OK;
}
