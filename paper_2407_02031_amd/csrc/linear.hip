// A linear layer with bias, activation and residual, and its backward pass.
//
//   z = x W^T + bias,  y = act(z) + residual
//   dz = dy act'(z):  dx = dz W,  dW = dz^T x,  dbias = sum_m dz
//
// The products run on the projections' tiles (gemm_tile.hpp): forward with the activation in the epilogue; backward with operands
// whose rows are the reduction's, which the transposing LDS read turns on the way into the registers, so that nothing is
// transposed in memory.  dz is formed once, in front of the products, by a kernel that sums its columns in fp32 too.
//
// Measured (kernels alone, three sets of inputs in turn; least and mean), 8192 rows, N = 5120, K = 1280: forward with GELU and z kept 115 to 121 us, 890 to 940 TFLOP/s; backward dz 47 to
// 50 us (252 MB, 5.0 to 5.4 TB/s), both products 192 to 208 (215 GFLOP, 1030 to 1120 TFLOP/s), what they left in parts 5.  1976 rows, N = 1280, K = 5120, fp32 with residual 37 to 39 us,
// 660 to 690 TFLOP/s: bound by what a CU draws of its one tile's operands.  One row, N = 5120, K = 1280 5.6 to 5.9 us, 2.2 to 2.3 TB/s: a launch and one trip to HBM.
// Backward of few rows, N = 5120, K = 1280, cold: 1 row 21.4 us (dx alone 13.8), 16 22.1, 64 24.0, 128 26.9: the weights come in and their gradient goes out at 1.1 to 1.2 TB/s, behind dz and
// ahead of the sum of dx's parts.
#include "gemm_tile.hpp"
#include "rows.hpp"

#include <string.h>
#include <algorithm>

namespace sd {

// ---------------------------------------------------------------------------------------
// dz and its column sums.  Bound by HBM (dy and z in, dz out).  CT threads have eight columns each; the NT / CT groups of them take rows in turn, four at
// a time in flight.  The sums of a workgroup's rows go to sums[row block] (where there is one row block, to the result itself).
// dz is rounded to bf16, once, whatever the types of dy and of dW (the sums are of what it was before): that is what the matrix cores multiply with x and W, which are bf16 themselves.  It
// is off by up to 2^-8 of each term; against 64 bits a bf16 gradient's error grows from 0.0017 of it, its own rounding, to 0.0023, and an fp32 dW has 0.0017 of it.  Two bf16 halves of dz would
// take both products twice (192 us more for 8192 x 5120 x 1280).  Its rows are Np elements long, N rounded up to a multiple of 8, with zeros behind N.
// ---------------------------------------------------------------------------------------
template <class D, bool STORE, bool SUMS, int CT, int NT>
__global__ __launch_bounds__(NT) void dz_kernel(const D* __restrict__ dy, const uint16_t* __restrict__ z, int act, uint16_t* __restrict__ dz, float* __restrict__ sums, int M, int N, int Np, int rows, int blocks) {
    constexpr int SUB = NT / CT, BATCH = 4;
    constexpr int PARTS = CT < 64 ? NT / 64 : SUB;          // sums of a column that meet in LDS
    __shared__ f32x8 sh[(PARTS - 1) * CT];
    const int t = threadIdx.x % CT, sub = threadIdx.x / CT;
    const int cols = (int)blockIdx.x / blocks, block = (int)blockIdx.x - cols * blocks;
    const int c = (cols * CT + t) * 8;
    const int64_t r0 = (int64_t)block * rows + sub;
    const int64_t r1 = min((int64_t)M, ((int64_t)block + 1) * rows);
    const bool whole = c + 8 <= N;
    const f32x4 zero = {0.f, 0.f, 0.f, 0.f};
    f32x8 sum = {zero, zero};
    const __bf16* const zb = reinterpret_cast<const __bf16*>(z);
    __bf16* const out = reinterpret_cast<__bf16*>(dz);
    // A row's last piece, where eight do not divide it, begins earlier, at N - 8: what it has in common with its neighbour's is written
    // twice, the same, and counted in the neighbour's sums alone.
    const int at = whole ? c : N - 8;
    auto all = [&](auto kind) {
        constexpr int KIND = decltype(kind)::value;
        auto slope = [&](f32x8 g, const f32x8& v) {
            if (KIND != SD_ACT_NONE)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    g.lo[e] *= act_slope<KIND>(v.lo[e]);
                    g.hi[e] *= act_slope<KIND>(v.hi[e]);
                }
            if (SUMS) {
                sum.lo += g.lo;
                sum.hi += g.hi;
            }
            return g;
        };
        if (N >= 8 && c < Np) {
            for (int64_t r = r0; r < r1; r += SUB * BATCH) {
                f32x8 g[BATCH], v[BATCH];
#pragma unroll
                for (int i = 0; i < BATCH; ++i) {
                    const int64_t o = min(r + i * SUB, r1 - 1) * N + at;
                    g[i] = load8(dy + o);
                    if (KIND != SD_ACT_NONE) v[i] = load8(zb + o);
                }
#pragma unroll
                for (int i = 0; i < BATCH; ++i)
                    if (r + i * SUB < r1) {
                        g[i] = slope(g[i], v[i]);
                        if (STORE) store8(out + (r + i * SUB) * Np + at, g[i]);
                    }
            }
        } else if (c < Np) {
            for (int64_t r = r0; r < r1; r += SUB) {
                f32x8 g = {zero, zero}, v = g;
#pragma unroll
                for (int e = 0; e < 7; ++e)
                    if (e < N) {
                        const float d = (float)dy[r * N + e], w = KIND != SD_ACT_NONE ? (float)zb[r * N + e] : 0.f;
                        if (e < 4) g.lo[e & 3] = d, v.lo[e & 3] = w;
                        else g.hi[e & 3] = d, v.hi[e & 3] = w;
                    }
                g = slope(g, v);
                if (STORE) store8(out + r * Np, g);
            }
        }
    };
    switch (act) {
    case SD_ACT_GELU: all(std::integral_constant<int, SD_ACT_GELU>()); break;
    case SD_ACT_GELU_TANH: all(std::integral_constant<int, SD_ACT_GELU_TANH>()); break;
    case SD_ACT_SILU: all(std::integral_constant<int, SD_ACT_SILU>()); break;
    case SD_ACT_RELU: all(std::integral_constant<int, SD_ACT_RELU>()); break;
    default: all(std::integral_constant<int, SD_ACT_NONE>());
    }
    if (STORE && N >= 8 && !whole && c < Np)
        for (int64_t r = r0; r < r1; r += SUB)
            for (int e = N; e < Np; ++e) dz[r * Np + e] = 0;
    if (SUMS) {
        int part = sub;
        if constexpr (CT < 64) {       // the rows of a wavefront
#pragma unroll
            for (int o = CT; o < 64; o *= 2)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    sum.lo[e] += __shfl_xor(sum.lo[e], o);
                    sum.hi[e] += __shfl_xor(sum.hi[e], o);
                }
            part = threadIdx.x >> 6;
        }
        if (part && (CT >= 64 || (threadIdx.x & 63) < CT)) sh[(part - 1) * CT + t] = sum;
        __syncthreads();
        if (threadIdx.x >= CT) return;
#pragma unroll
        for (int w = 0; w < PARTS - 1; ++w) {
            sum.lo += sh[w * CT + t].lo;
            sum.hi += sh[w * CT + t].hi;
        }
        float* const to = sums + (int64_t)block * N + c;
        if (whole) {
            store4(to, sum.lo);
            store4(to + 4, sum.hi);
        } else {
            const int first = N >= 8 ? N - 8 : 0;
#pragma unroll
            for (int e = 0; e < 8; ++e)
                if (first + e >= c && first + e < N) to[first - c + e] = e < 4 ? sum.lo[e & 3] : sum.hi[e & 3];
        }
    }
}
// How dz is cut.  Few rows: 16 columns and all rows a workgroup, so that no sums of row blocks are left.  Else 512 columns (of 2048 a row's end leaves more idle: dz and a product
// of 8 columns, 8192 x 2560 54.7 / 47.9 us, 8192 x 1280 33.9 / 30.3) and as many rows as leave two workgroups a CU, 8 to 32.  (us, a whole backward pass to K = 640, few rows / else: 128 x 640 11.0 / 12.4, 300 x 317 12.9 / 13.3, 500 x 1280 17.2 / 19.0, 1003 x 640 17.2 / 17.5, and a launch less; of rows
// at odd addresses, whose pieces lie in two lines each, 500 x 317 15.7 / 14.5, 1003 x 317 21.6 / 18.0.)
struct DzCut {
    int ct, nt, rows;
    int64_t col_wgs, blocks;
    DzCut(int64_t M, int64_t N) {
        const int64_t Np = (N + 7) & ~7ll;
        const bool few = M <= 256 || (M <= (N % 8 ? 384 : 1024) && M * N <= (1 << 20));
        ct = few ? 2 : 64;
        nt = few ? 1024 : 256;
        col_wgs = (Np + ct * 8 - 1) / (ct * 8);
        const int64_t r = M * col_wgs / 512;
        rows = few ? 1024 : r >= 32 ? 32 : r >= 16 ? 16 : 8;
        blocks = (M + rows - 1) / rows;
    }
};

constexpr int GATED_DZ_THREADS = 256;
// ... of a gated layer's: 64 x 4 threads for any rows.  (Few rows in one block, as above, would take workgroups of 1024 threads whose registers do not hold two columns' sums of eight: all of the
// backward pass, us, these / those: one row of 1280 to 5120 27.6 / 40.5, 200 41 / 51, 77 of 640 to 640 12.0 / 16.1, 1000 of 640 to 64 17.3 / 23.1.)
struct GatedDzCut {
    int rows;
    int64_t col_wgs, blocks;
    GatedDzCut(int64_t M, int64_t N) {
        col_wgs = (N + 511) / 512;
        const int64_t r = M * col_wgs / 512;
        rows = r >= 32 ? 32 : r >= 16 ? 16 : 8;
        blocks = (M + rows - 1) / rows;
    }
};
// The same of a gated layer: dy [M, N] and z = [v, g] [M, 2 N] in, dz = [dy act(g), dy v act'(g)] [M, Np] out, Np 2 N rounded up to a multiple of 8; its column sums are 2 N.  Where N is
// no multiple of eight, accesses to the gate's half are aligned to an element alone.  Bound by HBM: 8192 x 5120 bf16 with SiLU 70 to 72 us (420 MB, 5.8 to 6.0 TB/s).  dz is rounded to bf16 as above.
// PAST: a large z is read past the caches, which dz has to itself then (all of the backward pass, us, past / through: 8192 x 1280 to 5120 456 / 463, 8192 x 640 to 2560 151 / 157, 4096 x 1280 to 5120 231.7 / 233.4;
// but 2048 135.5 / 134.8 and 2048 x 640 to 2560 50.6 / 49.4).
template <class D, bool STORE, bool SUMS, bool PAST>
__global__ __launch_bounds__(GATED_DZ_THREADS) void gated_dz_kernel(const D* __restrict__ dy, const uint16_t* __restrict__ z, int act, uint16_t* __restrict__ dz, float* __restrict__ sums, int M, int N, int Np, int rows, int blocks) {
    constexpr int CT = 64, SUB = GATED_DZ_THREADS / CT, BATCH = 2;
    __shared__ f32x8 sh[2 * (SUB - 1) * CT];
    const int t = threadIdx.x % CT, sub = threadIdx.x / CT;
    const int cols = (int)blockIdx.x / blocks, block = (int)blockIdx.x - cols * blocks;
    const int c = (cols * CT + t) * 8;
    const int64_t r0 = (int64_t)block * rows + sub;
    const int64_t r1 = min((int64_t)M, ((int64_t)block + 1) * rows);
    const f32x4 zero = {0.f, 0.f, 0.f, 0.f};
    f32x8 sv = {zero, zero}, sg = sv;
    const __bf16* const zb = reinterpret_cast<const __bf16*>(z);
    __bf16* const out = reinterpret_cast<__bf16*>(dz);
    const int at = c + 8 <= N ? c : N - 8;        // (as in dz_kernel)
    auto load_z = [](const __bf16* p) {
        if constexpr (!PAST) return load8(p);
        const bf16x8u v = __builtin_nontemporal_load(reinterpret_cast<const bf16x8u*>(p));
        return f32x8{{(float)v[0], (float)v[1], (float)v[2], (float)v[3]}, {(float)v[4], (float)v[5], (float)v[6], (float)v[7]}};
    };
    auto all = [&](auto kind) {
        constexpr int KIND = decltype(kind)::value;
        auto one = [&](f32x4& d, f32x4& v, const f32x4& g) {        // d <- dy act(g), v <- dy v act'(g)
            f32x4 a[1] = {g};
            apply_act(KIND, a);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                v[e] *= d[e] * act_slope<KIND>(g[e]);
                d[e] *= a[0][e];
            }
        };
        auto both = [&](f32x8& d, f32x8& v, const f32x8& g) {
            one(d.lo, v.lo, g.lo);
            one(d.hi, v.hi, g.hi);
            if (SUMS) {
                sv.lo += d.lo;
                sv.hi += d.hi;
                sg.lo += v.lo;
                sg.hi += v.hi;
            }
        };
        if (N >= 8 && c < N) {
            for (int64_t r = r0; r < r1; r += SUB * BATCH) {
                f32x8 d[BATCH], v[BATCH], g[BATCH];
#pragma unroll
                for (int i = 0; i < BATCH; ++i) {
                    const int64_t row = min(r + i * SUB, r1 - 1);
                    d[i] = load8(dy + row * N + at);
                    v[i] = load_z(zb + row * 2 * N + at);
                    g[i] = load_z(zb + row * 2 * N + N + at);
                }
#pragma unroll
                for (int i = 0; i < BATCH; ++i)
                    if (r + i * SUB < r1) {
                        both(d[i], v[i], g[i]);
                        if (STORE) {
                            store8(out + (r + i * SUB) * Np + at, d[i]);
                            store8(out + (r + i * SUB) * Np + N + at, v[i]);
                        }
                    }
            }
        } else if (c < N) {
            for (int64_t r = r0; r < r1; r += SUB) {
                f32x8 d = {zero, zero}, v = d, g = d;
#pragma unroll
                for (int e = 0; e < 7; ++e)
                    if (e < N) {
                        const float dd = (float)dy[r * N + e], vv = (float)zb[r * 2 * N + e], gg = (float)zb[r * 2 * N + N + e];
                        if (e < 4) d.lo[e & 3] = dd, v.lo[e & 3] = vv, g.lo[e & 3] = gg;
                        else d.hi[e & 3] = dd, v.hi[e & 3] = vv, g.hi[e & 3] = gg;
                    }
                both(d, v, g);
                if (STORE)
#pragma unroll
                    for (int e = 0; e < 7; ++e)
                        if (e < N) {
                            out[r * Np + e] = (__bf16)(e < 4 ? d.lo[e & 3] : d.hi[e & 3]);
                            out[r * Np + N + e] = (__bf16)(e < 4 ? v.lo[e & 3] : v.hi[e & 3]);
                        }
            }
        }
    };
    switch (act) {
    case SD_ACT_GELU: all(std::integral_constant<int, SD_ACT_GELU>()); break;
    case SD_ACT_GELU_TANH: all(std::integral_constant<int, SD_ACT_GELU_TANH>()); break;
    case SD_ACT_SILU: all(std::integral_constant<int, SD_ACT_SILU>()); break;
    case SD_ACT_RELU: all(std::integral_constant<int, SD_ACT_RELU>()); break;
    default: all(std::integral_constant<int, SD_ACT_NONE>());
    }
    if (STORE && c < N && c + 8 >= N)
        for (int64_t r = r0; r < r1; r += SUB)
            for (int e = 2 * N; e < Np; ++e) dz[r * Np + e] = 0;
    if (SUMS) {
        if (sub) {
            sh[(sub - 1) * 2 * CT + t] = sv;
            sh[(sub - 1) * 2 * CT + CT + t] = sg;
        }
        __syncthreads();
        if (threadIdx.x >= CT || c >= N) return;
#pragma unroll
        for (int w = 0; w < SUB - 1; ++w) {
            sv.lo += sh[w * 2 * CT + t].lo;
            sv.hi += sh[w * 2 * CT + t].hi;
            sg.lo += sh[w * 2 * CT + CT + t].lo;
            sg.hi += sh[w * 2 * CT + CT + t].hi;
        }
        const int first = c + 8 <= N ? c : N >= 8 ? N - 8 : 0;
        float* const to = sums + (int64_t)block * 2 * N + first;
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (first + e >= c && first + e < N) {
                to[e] = e < 4 ? sv.lo[e & 3] : sv.hi[e & 3];
                to[N + e] = e < 4 ? sg.lo[e & 3] : sg.hi[e & 3];
            }
    }
}

// ---------------------------------------------------------------------------------------
// What is left in parts: dx, dW (as many fp32 matrices as their reductions were cut into) and dbias (a row for every
// row block of dz), each added up in order, in one launch.  256 threads: 1024 elements of a matrix, or 16 columns of dbias.
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
    __shared__ float sh[4][16];
    const int c = wg * 16 + (threadIdx.x & 15), at = min(c, a.N - 1);
    float s = 0.f;
#pragma unroll 8
    for (int b = threadIdx.x >> 4; b < a.blocks; b += 16) s += a.sums[(int64_t)b * a.N + at];
    s += __shfl_xor(s, 16);
    s += __shfl_xor(s, 32);
    if ((threadIdx.x & 63) < 16) sh[threadIdx.x >> 6][threadIdx.x & 15] = s;
    __syncthreads();
    if (threadIdx.x < 16 && c < a.N) a.dbias[c] = s + sh[1][threadIdx.x] + sh[2][threadIdx.x] + sh[3][threadIdx.x];
}
static Parts parts_of(const float* parts, void* out, bool f32, int64_t n, int count) { return Parts{parts, out, n, count, f32, (int32_t)((n / 4 + 255) / 256)}; }
static int launch_part_sums(PartSums& a, hipStream_t stream) {
    const int64_t wgs = (int64_t)a.m[0].wgs + a.m[1].wgs + (a.dbias ? (a.N + 15) / 16 : 0);
    SD_REQUIRE(wgs < (1 << 24), SD_EUNSUPPORTED, "linear_bwd: gradients of 2^34 elements and more in parts, or of nothing");      // (threads of a launch stay below 2^32)
    if (wgs == 0 || SD_DRY_RUN("part sums; ")) return SD_OK;
    hipLaunchKernelGGL(part_sums_kernel, dim3((unsigned)wgs), dim3(256), 0, stream, a);
    SD_HIP_CHECK(hipGetLastError());
    return SD_OK;
}

// ---------------------------------------------------------------------------------------
// products
// ---------------------------------------------------------------------------------------
template <int BM, int BN, int WGM, int WGN, int STAGES>
static int launch_act(GemmGroup& g, hipStream_t stream) {
    GemmProblem& P = g.p[0];
    P.tiles_m = (P.Mp + BM - 1) / BM;
    P.tiles_n = (P.N + BN - 1) / BN;
    g.total_tiles = P.tiles_m * P.tiles_n;
    const bool guard = P.K0 % 64 != 0;
    if (SD_DRY_RUN("gemm act %dx%d/%d waves/%d stages%s%s; ", BM, BN, WGM * WGN, STAGES, guard ? " guard" : "", P.z && gemm_z_past<BN / WGN / 16>(P.Mp, P.ldy) ? dry_detail(", z past the caches") : ""))
        return SD_OK;
    const dim3 grid((g.total_tiles + 7) & ~7), block(64 * WGM * WGN);
    if (guard) hipLaunchKernelGGL((gemm_kernel<BM, BN, 64, WGM, WGN, STAGES, false, true, false, GemmAct>), grid, block, 0, stream, g, GemmAct{});
    else hipLaunchKernelGGL((gemm_kernel<BM, BN, 64, WGM, WGN, STAGES, false, false, false, GemmAct>), grid, block, 0, stream, g, GemmAct{});
    SD_HIP_CHECK(hipGetLastError());
    return SD_OK;
}
// Tiles of a linear layer with more of them than one round of small ones: the launch is taken to last its rounds times what a round takes, us, a first part and a part for every step of 64.
// Each of the five is the fastest of some launches (us, z kept, cold, it / the next: 64x128 4096x640x2560 44.0 / 50.3, 128x128 16384x1920x640 67.4 / 73.3, 128x160 8192x1280x5120 130 /
// 164, 256x128 8192x1920x640 40.2 / 43.7, 128x256 2960x5120x1280 52.6 / 56.5).  Of 49 launches of 1000 to 16384 rows 38 get the fastest or one within 3 % of it; the mean of all is 2 %
// above.  The others are those that the model knows too little of: it has no term for the bytes of y and z, which count where K is short, and takes 128x256 and 256x128 for nearly the
// same (taken / fastest: 8192x1920x640 128x256 50.6 / 40.2, 16384x1920x640 128x256 80.8 / 67.4, 2960x1920x640 128x256 23.7 / 21.1, 8192x5120x1280 128x256 138 / 130, 16384x1280x1280 128x160
// 85.8 / 80.2).
static int launch_large(GemmGroup& g, hipStream_t stream) {
    struct Tile { int bm, bn, slots; float step, rest; };
    static const Tile tiles[5] = {{64, 128, 512, 0.85f, 4.f}, {128, 128, 512, 1.12f, 7.f}, {128, 160, 512, 1.45f, 9.f}, {256, 128, 256, 1.02f, 6.f}, {128, 256, 256, 1.0f, 6.f}};
    const GemmProblem& P = g.p[0];
    int best = 0;
    float least = 0.f;
    for (int i = 0; i < 5; ++i) {
        const Tile& t = tiles[i];
        const int64_t n = (int64_t)((P.Mp + t.bm - 1) / t.bm) * ((P.N + t.bn - 1) / t.bn);
        const float us = (float)((n + t.slots - 1) / t.slots) * ((float)((P.K0 + 63) / 64) * t.step + t.rest);
        if (i == 0 || us < least) best = i, least = us;
    }
    switch (best) {
    case 0: return launch_act<64, 128, 2, 2, 3>(g, stream);
    case 1: return launch_act<128, 128, 2, 2, 2>(g, stream);
    case 2: return launch_act<128, 160, 2, 2, 2>(g, stream);
    case 3: return launch_act<256, 128, 4, 2, 3>(g, stream);
    default: return launch_act<128, 256, 2, 4, 3>(g, stream);
    }
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

// Two kernels: 256x128 tiles of eight wavefronts, three stages, one workgroup a CU, and 64x128 ones of four, two a CU.  (Of the former, us, both products, 128x128 tiles of four
// wavefronts two a CU / these: M = 8192, N = 5120, K = 1280 253 / 229, 2048 x 5120 x 1280 77.3 / 75.9, 8192 x 640 x 640 34.4 / 32.6; 256x256 tiles 262, 85, 47.  The latter take
// small products, which then need fewer cuts or none: 300 x 515 x 1024 8.0 us where the larger tiles with three parts took 15.8.)
constexpr int BWD_CUS = 256, BWD_PARTS = GEMM_MAX_PROBLEMS / 2;
constexpr int BWD_BM = 256, BWD_SMALL_BM = 64, BWD_BN = 128;
// How a product's reduction is cut: the first `whole` rows of the result not at all, the others into `parts` sums over consecutive steps of 64, which
// part_sums adds up.
struct BwdCut {
    int64_t rows, cols, steps, tiles_n, tiles;
    int64_t whole;
    int parts;
    BwdCut(int64_t r, int64_t c, int64_t depth, int bm) : rows(r), cols(c), steps((depth + 63) / 64), tiles_n((c + BWD_BN - 1) / BWD_BN), tiles((r + bm - 1) / bm * tiles_n), whole(r), parts(1) {}
    void all_in(int p) {
        parts = p;
        whole = p > 1 ? 0 : rows;
    }
    size_t bytes() const { return parts > 1 ? (size_t)parts * (rows - whole) * cols * 4 : 0; }
};
// Tiles of two kinds on so many slots, the longer ones first: `an` of as steps, dealt evenly, then bn of bs where one is free
template <class I>
struct BwdRounds {
    I q, r, as, bn, bs, slots;
    BwdRounds(int64_t an, int64_t as_, int64_t bn_, int64_t bs_, int slots_) : q((I)an / slots_), r((I)an % slots_), as((I)as_), bn((I)bn_), bs((I)bs_), slots(slots_) {}
    // of the second kind done after d steps
    I done(I d) const { return r * (std::max<I>(d - (q + 1) * as, 0) / bs) + (slots - r) * (std::max<I>(d - q * as, 0) / bs); }
    // steps until all are done
    I until() const {
        I d = std::max<I>((q + (r > 0)) * as, (r * as + q * slots * as + bn * bs + slots - 1) / slots);
        while (done(d) < bn) d += std::min<I>(bs - std::max<I>(d - q * as, 0) % bs, bs - std::max<I>(d - (q + 1) * as, 0) % bs);
        return d;
    }
};
// From the sizes alone, as for both products: a gradient's bits do not depend on which others are wanted.
struct BwdPlan {
    BwdCut x, w;
    bool small;
    bool w_first;                  // the product of the longer sums goes first
    BwdPlan(int64_t M, int64_t N, int64_t K) : x(M, K, N, BWD_BM), w(N, K, M, BWD_BM), small(false) {
        // What a choice takes, us: its steps and its first loads and stores (a step of the small tiles waits less where they have a CU to themselves), the parts written and read again at
        // 4 TB/s, and the launch that adds them up
        float least = 0.f;
        int px = 0, pw = 0;
        for (int sm = 1; sm >= 0; --sm) {
            const int bm = sm ? BWD_SMALL_BM : BWD_BM;
            const BwdCut cx(M, K, N, bm), cw(N, K, M, bm);
            const int slots = sm ? 2 * BWD_CUS : BWD_CUS;
            if (sm && cx.tiles + cw.tiles > 2 * slots) continue;
            // (in 32 bits where they do, which is cheaper)
            const bool narrow = cx.tiles * cx.steps + cw.tiles * cw.steps < (1 << 26);
            for (int a = 1; a <= BWD_PARTS; a += a >= 4 ? 2 : 1)
                for (int b = 1; b <= BWD_PARTS; b += b >= 4 ? 2 : 1) {
                    if ((a > 1 && cx.steps < 4 * a) || (b > 1 && cw.steps < 4 * b)) break;
                    const int64_t sx = (cx.steps + a - 1) / a, sw = (cw.steps + b - 1) / b, nx = cx.tiles * a, nw = cw.tiles * b;
                    const bool wl = sw > sx;
                    const int64_t an = wl ? nw : nx, as = wl ? sw : sx, bn = wl ? nx : nw, bs = wl ? sx : sw;
                    const int64_t d = narrow ? BwdRounds<int32_t>(an, as, bn, bs, slots).until() : BwdRounds<int64_t>(an, as, bn, bs, slots).until();
                    const float parts = (a > 1 ? (float)a * M * K : 0.f) + (b > 1 ? (float)b * N * K : 0.f);
                    const float us = (sm ? d * (nx + nw > BWD_CUS ? 0.85f : 0.57f) + 4.f : d * 0.9f + 6.f) + (parts > 0 ? 6.f + parts * 2e-6f : 0.f);
                    if (px == 0 || us < least) least = us, px = a, pw = b, small = sm;
                }
        }
        if (small) {
            x = BwdCut(M, K, N, BWD_SMALL_BM);
            w = BwdCut(N, K, M, BWD_SMALL_BM);
        }
        x.all_in(px);
        w.all_in(pw);
        w_first = w.steps * px > x.steps * pw;
        // The other product's tiles fill up what the first one's leave; where the last of them would be a round of few, they are cut in four.  (M = 8192, N =
        // 5120, K = 1280: 200 tiles of 128 steps, 320 of 80; the last 8 of these cut 201 us, not cut 229.)
        BwdCut &a = w_first ? w : x, &b = w_first ? x : w;
        if (!small && b.parts == 1 && b.steps >= 16) {
            const BwdRounds<int64_t> t(a.tiles * a.parts, (a.steps + a.parts - 1) / a.parts, b.tiles, b.steps, BWD_CUS);
            const int64_t share = (a.tiles * a.steps + b.tiles * b.steps + BWD_CUS - 1) / BWD_CUS, aim = std::max(share, (t.q + (t.r > 0)) * t.as) + share / 20 + 4;
            const int64_t left = (b.tiles - std::min(t.done(aim), b.tiles) + b.tiles_n - 1) / b.tiles_n;     // rows of tiles
            // a cut tile's parts are 0.5 MB written and read, 0.065 us of the chip's memory traffic each; a step takes 0.9 us
            if (left > 0 && t.until() > aim && left * b.tiles_n * 4 * 0.065 < (t.until() - aim) * 0.9) {
                b.parts = 4;
                b.whole = std::max<int64_t>(0, (b.rows + BWD_BM - 1) / BWD_BM - left) * BWD_BM;
            }
        }
    }
};
// out [rows, cols] = P^T Q (pt) or P Q over `depth`; p [depth, rows] or [rows, depth], q [depth, cols]
static void push_product(GemmGroup& g, bool pt, const uint16_t* p, int64_t ldp, const uint16_t* q, int64_t ldq, void* out, bool out_f32, const BwdCut& c, int depth, float* parts) {
    auto push = [&](int64_t row, int64_t rows, int64_t s0, int64_t s1, void* y, bool f32) {
        if (rows <= 0) return;
        GemmProblem& P = g.p[g.n++];
        P.p0 = p + (pt ? s0 * 64 * ldp + row : row * ldp + s0 * 64);
        P.ldp0 = ldp;
        P.q0 = q + s0 * 64 * ldq;
        P.ldq0 = ldq;
        P.Mp = (int32_t)rows;
        P.N = (int32_t)c.cols;
        P.K0 = (int32_t)(std::min<int64_t>(depth, s1 * 64) - s0 * 64);
        P.alpha = 1.f;
        P.ldy = c.cols;
        P.y = y;
        P.y_f32 = f32;
    };
    push(0, c.whole, 0, c.steps, out, out_f32);
    for (int i = 0; i < c.parts && c.parts > 1; ++i) push(c.whole, c.rows - c.whole, c.steps * i / c.parts, c.steps * (i + 1) / c.parts, parts + (size_t)i * (c.rows - c.whole) * c.cols, true);
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
// Few rows (one token's, a guidance pair's, a short text's).  A workgroup has 16 MB rows and 16 NB columns, and its eight wavefronts every eighth step of 32 of the
// reduction each; they bring the rows of x and W straight into the registers as MFMA operands, so that all of a short reduction's loads are in flight at once, and meet
// in LDS when they are done.  Bound by the weights, which come in once per 16 MB rows, and one trip to HBM.
// ---------------------------------------------------------------------------------------
constexpr int ROWS_NW = 8;
template <int MB, int NB, int U>
__global__ __launch_bounds__(64 * ROWS_NW) void linear_rows_kernel(const uint16_t* __restrict__ x, const uint16_t* __restrict__ W, const uint16_t* __restrict__ bias, int act, const void* res,
                                                                   void* y, int f32, uint16_t* __restrict__ z, int M, int N, int K) {
    constexpr int NW = ROWS_NW, BLOCKS = MB * NB, PER = (BLOCKS + NW - 1) / NW;
    __shared__ f32x4 sh[NW * BLOCKS * 64];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int l16 = lane & 15, quad = lane >> 4;
    const int n0 = blockIdx.x * (16 * NB), m0 = blockIdx.y * (16 * MB);
    const uint16_t *wr[NB], *xr[MB];
    f32x4 acc[MB][NB];
#pragma unroll
    for (int n = 0; n < NB; ++n) wr[n] = W + (int64_t)min(n0 + n * 16 + l16, N - 1) * K + quad * 8;
#pragma unroll
    for (int m = 0; m < MB; ++m) {
        xr[m] = x + (int64_t)min(m0 + m * 16 + l16, M - 1) * K + quad * 8;
#pragma unroll
        for (int n = 0; n < NB; ++n) acc[m][n] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
    const int steps = (K + 31) / 32;
    const u32x4 none = {0u, 0u, 0u, 0u};
    u32x4 wf[U][NB], xf[U][MB];
    auto fetch = [&](int s0) {
#pragma unroll
        for (int i = 0; i < U; ++i) {
            const int k = (s0 + i * NW) * 32;
            const bool in = k + quad * 8 < K;         // (a chunk of eight is whole or not there)
#pragma unroll
            for (int n = 0; n < NB; ++n) wf[i][n] = in ? *reinterpret_cast<const u32x4*>(wr[n] + k) : none;
#pragma unroll
            for (int m = 0; m < MB; ++m) xf[i][m] = in ? *reinterpret_cast<const u32x4*>(xr[m] + k) : none;
        }
    };
    fetch(wave);
    // what the epilogue adds, behind the first loads: wavefront w finishes blocks w, w + 8, ..., a lane has four columns of one row.  (Asked for there, one more trip to HBM.)
    f32x4 bv[PER], rv[PER];
    auto place = [&](int i, int& row, int& col) {
        const int b = wave + i * NW;
        row = m0 + b / NB * 16 + l16;
        col = n0 + b % NB * 16 + quad * 4;
        return b < BLOCKS && row < M && col < N;
    };
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        bv[i] = rv[i] = f32x4{0.f, 0.f, 0.f, 0.f};
        int row, col;
        if (!place(i, row, col)) continue;
        const int64_t at = (int64_t)row * N + col;
        const __bf16* const bb = reinterpret_cast<const __bf16*>(bias) + col;
        if (col + 4 <= N) {
            if (bias) bv[i] = load4(bb);
            if (res) rv[i] = f32 ? load4(static_cast<const float*>(res) + at) : load4(static_cast<const __bf16*>(res) + at);
        } else
#pragma unroll
            for (int e = 0; e < 3; ++e)
                if (col + e < N) {
                    if (bias) bv[i][e] = (float)bb[e];
                    if (res) rv[i][e] = f32 ? static_cast<const float*>(res)[at + e] : (float)static_cast<const __bf16*>(res)[at + e];
                }
    }
    for (int s0 = wave;;) {
#pragma unroll
        for (int i = 0; i < U; ++i)
#pragma unroll
            for (int m = 0; m < MB; ++m)
#pragma unroll
                for (int n = 0; n < NB; ++n)
                    acc[m][n] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, wf[i][n]), __builtin_bit_cast(bf16x8, xf[i][m]), acc[m][n], 0, 0, 0);
        s0 += NW * U;
        if (s0 >= steps) break;
        fetch(s0);
    }
#pragma unroll
    for (int b = 0; b < BLOCKS; ++b) sh[(wave * BLOCKS + b) * 64 + lane] = acc[b / NB][b % NB];
    __syncthreads();
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        int row, col;
        if (!place(i, row, col)) continue;
        const int b = wave + i * NW;
        f32x4 v[1] = {sh[b * 64 + lane]};
#pragma unroll
        for (int w = 1; w < NW; ++w) v[0] += sh[(w * BLOCKS + b) * 64 + lane];
        v[0] += bv[i];
        const f32x4 pre = v[0];
        apply_act(act, v);
        v[0] += rv[i];
        const int64_t at = (int64_t)row * N + col;
        __bf16* const zp = reinterpret_cast<__bf16*>(z) + at;
        if (col + 4 <= N) {
            if (z) store4(zp, pre);
            if (f32) store4(static_cast<float*>(y) + at, v[0]);
            else store4(static_cast<__bf16*>(y) + at, v[0]);
        } else
#pragma unroll
            for (int e = 0; e < 3; ++e)
                if (col + e < N) {
                    if (z) zp[e] = (__bf16)pre[e];
                    if (f32) static_cast<float*>(y)[at + e] = v[0][e];
                    else static_cast<__bf16*>(y)[at + e] = (__bf16)v[0][e];
                }
    }
}
template <int MB, int NB, int U>
static int launch_rows(const uint16_t* x, const uint16_t* W, const uint16_t* bias, int act, const void* res, void* y, int f32, uint16_t* z, int M, int N, int K, hipStream_t stream) {
    if (SD_DRY_RUN("linear rows %dx%d; ", 16 * MB, 16 * NB)) return SD_OK;
    hipLaunchKernelGGL((linear_rows_kernel<MB, NB, U>), dim3((N + 16 * NB - 1) / (16 * NB), (M + 16 * MB - 1) / (16 * MB)), dim3(64 * ROWS_NW), 0, stream, x, W, bias, act, res, y, f32, z, M, N, K);
    SD_HIP_CHECK(hipGetLastError());
    return SD_OK;
}
constexpr int LINEAR_MAX_M = 1 << 28, LINEAR_MAX_NK = 1 << 22;
static int linear_sizes(const char* who, int M, int N, int K, int act, int y_dtype) {
    SD_REQUIRE(M >= 0 && N >= 0, SD_EINVAL, "%s: M=%d N=%d", who, M, N);
    SD_REQUIRE(K > 0 && K % 8 == 0, SD_EUNSUPPORTED, "%s: K=%d is not a positive multiple of 8", who, K);
    // (threads of a launch stay below 2^32)
    SD_REQUIRE(M < LINEAR_MAX_M && N < LINEAR_MAX_NK && K < LINEAR_MAX_NK, SD_EUNSUPPORTED, "%s: M=%d N=%d K=%d (M below 2^28, N and K below 2^22)", who, M, N, K);
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
        sums = (size_t)DzCut(M, N).blocks * N * 4;
        const BwdPlan p(M, N, K);
        dx_parts = p.x.bytes();
        dw_parts = p.w.bytes();
    }
    size_t total() const { return round_up(dz, 256) + round_up(sums, 256) + round_up(dx_parts, 256) + round_up(dw_parts, 256) + 256; }
};

// dx = dz W and dW = dz^T x, dz with rows of Np elements, and what `left` holds besides of what is in parts
static int launch_products(const uint16_t* dz, int Np, const uint16_t* x, const uint16_t* W, uint16_t* dx, void* dW, int dw_dtype, float* dx_parts, float* dw_parts, PartSums& left, int M, int N, int K,
                           const BwdPlan& plan, hipStream_t s) {
    if (dx || dW) {
        GemmGroup g;
        memset(&g, 0, sizeof(g));
        const bool dw_first = dW && (!dx || plan.w_first);
        auto push_dw = [&] {
            if (dW) push_product(g, true, dz, Np, x, K, dW, dw_dtype == SD_F32, plan.w, M, dw_parts);
        };
        if (dw_first) push_dw();
        const int dx_from = g.n;
        if (dx) push_product(g, false, dz, Np, W, K, dx, false, plan.x, N, dx_parts);
        const int dx_to = g.n;
        if (!dw_first) push_dw();
        const bool guard = (dW && M % 64 != 0) || (dx && N % 64 != 0);
        const int dw_from = dw_first ? 0 : dx_to, dw_to = dw_first ? dx_from : g.n;
        const int rc = plan.small ? launch_bwd<BWD_SMALL_BM, BWD_BN, 2, 2, 3>(g, dw_from, dw_to, guard, s) : launch_bwd<BWD_BM, BWD_BN, 4, 2, 3>(g, dw_from, dw_to, guard, s);
        if (rc) return rc;
        auto rest = [&](const BwdCut& c, const float* parts, void* out, bool f32) {
            return parts_of(parts, static_cast<char*>(out) + c.whole * c.cols * (f32 ? 4 : 2), f32, (c.rows - c.whole) * c.cols, c.parts);
        };
        if (dx && plan.x.parts > 1) left.m[0] = rest(plan.x, dx_parts, dx, false);
        if (dW && plan.w.parts > 1) left.m[1] = rest(plan.w, dw_parts, dW, dw_dtype == SD_F32);
    }
    return launch_part_sums(left, s);
}
// what sd_gated_linear_bwd carves out of its workspace
struct GatedBwdWs {
    size_t dz, sums, dx_parts, dw_parts;
    GatedBwdWs(int64_t M, int64_t N, int64_t K) {
        dz = (size_t)M * ((2 * N + 7) & ~7ll) * 2;
        sums = (size_t)GatedDzCut(M, N).blocks * 2 * N * 4;
        const BwdPlan p(M, 2 * N, K);
        dx_parts = p.x.bytes();
        dw_parts = p.w.bytes();
    }
    size_t total() const { return round_up(dz, 256) + round_up(sums, 256) + round_up(dx_parts, 256) + round_up(dw_parts, 256) + 256; }
};
constexpr int GATED_MAX_N = LINEAR_MAX_NK / 2;

}  // namespace sd

using namespace sd;

extern "C" int sd_linear_fwd(const uint16_t* x, const uint16_t* W, const uint16_t* bias, int32_t act, const void* residual, void* y, int32_t y_dtype, uint16_t* z,
                             int32_t M, int32_t N, int32_t K, void* stream) {
    int rc = linear_sizes("linear_fwd", M, N, K, act, y_dtype);
    if (rc || M == 0 || N == 0) return rc;
    SD_REQUIRE(x && W && y, SD_EINVAL, "linear_fwd: x, W or y is null");
    SD_REQUIRE(aligned16(x) && aligned16(W) && aligned16(bias) && aligned16(residual) && aligned16(y) && aligned16(z), SD_EINVAL, "linear_fwd: pointers must be 16-byte aligned");
    SD_REQUIRE(y != x && y != W && y != z && z != x && z != W && (!z || z != residual), SD_EINVAL, "linear_fwd: y or z in an input's place");
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
    // Up to 16 rows, and what the projections' one-round tiles do not take (their rule; K % 64, N % 4): straight from the weights, by the smallest tiles that are
    // one round.  (us, cold, these kernels / 64x128 tiles: 1 x 5120 x 1280 6.1 / 12.8, 1 x 1280 x 5120 9.5 / 38.4, 300 x 1280 x 1280 10.2 / 13.9, but 500 x 1280 x 1280, two rounds,
    // 17.9 / 14.8.)
    const int f32 = y_dtype == SD_F32;
    if (M <= 16) return launch_rows<1, 1, 6>(x, W, bias, act, residual, y, f32, z, M, N, K, s);
    P.set_act(act);
    P.z = z;
    if (gemm16_takes(g)) return launch_gemm16(g, s);
    const int64_t r32 = (M + 31) / 32, r64 = (M + 63) / 64, c16 = (N + 15) / 16, c32 = (N + 31) / 32;
    if (r32 * c16 <= 256) return launch_rows<2, 1, 6>(x, W, bias, act, residual, y, f32, z, M, N, K, s);
    if (r32 * c32 <= 256) return launch_rows<2, 2, 4>(x, W, bias, act, residual, y, f32, z, M, N, K, s);
    if (r64 * c32 <= 256) return launch_rows<4, 2, 3>(x, W, bias, act, residual, y, f32, z, M, N, K, s);
    return launch_large(g, s);
}

extern "C" size_t sd_linear_bwd_workspace_bytes(int32_t M, int32_t N, int32_t K) {
    if (M <= 0 || N <= 0 || K <= 0 || M >= LINEAR_MAX_M || N >= LINEAR_MAX_NK || K >= LINEAR_MAX_NK) return 256;      // (nothing to do, or refused)
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
    for (const void* const out : {static_cast<const void*>(dx), static_cast<const void*>(dW), static_cast<const void*>(dbias)})
        SD_REQUIRE(!out || (out != dy && out != x && out != W && out != z), SD_EINVAL, "linear_bwd: a gradient in an input's place");
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
    const int Np = (N + 7) & ~7;
    const DzCut cut(M, N);
    const int blocks = (int)cut.blocks;
    // dz is dy itself where nothing changes it on the way
    const bool plain = !zin && y_dtype == SD_BF16 && Np == N;
    const bool store = (dx || dW) && !plain;
    if ((store || dbias) && !SD_DRY_RUN("dz%s%s; ", store ? "" : " sums only", dbias ? "" : " no sums")) {
        const dim3 grid((unsigned)(cut.blocks * cut.col_wgs));
        float* const to = blocks == 1 ? dbias : sums;
        auto run = [&](auto* t, auto ct, auto nt) {
            using D = std::remove_pointer_t<decltype(t)>;
            constexpr int CT = decltype(ct)::value, NT = decltype(nt)::value;
            const D* const d = static_cast<const D*>(dy);
            if (store && dbias) hipLaunchKernelGGL((dz_kernel<D, true, true, CT, NT>), grid, dim3(NT), 0, s, d, zin, act, dzbuf, to, M, N, Np, cut.rows, blocks);
            else if (store) hipLaunchKernelGGL((dz_kernel<D, true, false, CT, NT>), grid, dim3(NT), 0, s, d, zin, act, dzbuf, to, M, N, Np, cut.rows, blocks);
            else hipLaunchKernelGGL((dz_kernel<D, false, true, CT, NT>), grid, dim3(NT), 0, s, d, zin, act, dzbuf, to, M, N, Np, cut.rows, blocks);
        };
        auto by_cut = [&](auto* t) {
            if (cut.ct == 2) run(t, std::integral_constant<int, 2>(), std::integral_constant<int, 1024>());
            else run(t, std::integral_constant<int, 64>(), std::integral_constant<int, 256>());
        };
        if (y_dtype == SD_F32) by_cut(static_cast<float*>(nullptr));
        else by_cut(static_cast<__bf16*>(nullptr));
        SD_HIP_CHECK(hipGetLastError());
    }
    if (dbias && blocks > 1) {
        left.sums = sums;
        left.dbias = dbias;
        left.blocks = blocks;
        left.N = N;
    }
    return launch_products(plain ? static_cast<const uint16_t*>(dy) : dzbuf, Np, x, W, dx, dW, dw_dtype, dx_parts, dw_parts, left, M, N, K, plan, s);
}

extern "C" size_t sd_gated_linear_bwd_workspace_bytes(int32_t M, int32_t N, int32_t K) {
    if (M <= 0 || N <= 0 || K <= 0 || M >= LINEAR_MAX_M || N >= GATED_MAX_N || K >= LINEAR_MAX_NK) return 256;      // (nothing to do, or refused)
    return GatedBwdWs(M, N, K).total();
}

extern "C" int sd_gated_linear_bwd(const void* dy, int32_t y_dtype, const uint16_t* x, const uint16_t* W, const uint16_t* z, int32_t act, uint16_t* dx, void* dW, int32_t dw_dtype,
                                   float* dbias, int32_t M, int32_t N, int32_t K, void* ws, size_t ws_bytes, void* stream) {
    SD_REQUIRE(N < GATED_MAX_N, SD_EUNSUPPORTED, "gated_linear_bwd: N=%d (below 2^21)", N);
    int rc = linear_sizes("gated_linear_bwd", M, N < 0 ? N : 2 * N, K, act, y_dtype);
    if (rc) return rc;
    SD_REQUIRE(dw_dtype == SD_BF16 || dw_dtype == SD_F32, SD_EINVAL, "gated_linear_bwd: dw_dtype=%d", dw_dtype);
    SD_REQUIRE(aligned16(dy) && aligned16(x) && aligned16(W) && aligned16(z) && aligned16(dx) && aligned16(dW) && aligned16(dbias), SD_EINVAL,
               "gated_linear_bwd: pointers must be 16-byte aligned");
    hipStream_t s = static_cast<hipStream_t>(stream);
    PartSums left;
    memset(&left, 0, sizeof(left));
    if (M == 0 || N == 0) {        // sums over nothing
        if (dx) left.m[0] = parts_of(nullptr, dx, false, (int64_t)M * K, 0);
        if (dW) left.m[1] = parts_of(nullptr, dW, dw_dtype == SD_F32, 2ll * N * K, 0);
        left.dbias = dbias;
        left.N = 2 * N;
        return launch_part_sums(left, s);
    }
    SD_REQUIRE(dy && z && (!dW || x) && (!dx || W), SD_EINVAL, "gated_linear_bwd: dy, z, x or W is null");
    for (const void* const out : {static_cast<const void*>(dx), static_cast<const void*>(dW), static_cast<const void*>(dbias)})
        SD_REQUIRE(!out || (out != dy && out != x && out != W && out != z), SD_EINVAL, "gated_linear_bwd: a gradient in an input's place");
    if (!dx && !dW && !dbias) return SD_OK;
    const size_t need = sd_gated_linear_bwd_workspace_bytes(M, N, K);
    SD_REQUIRE(ws && ws_bytes >= need && (reinterpret_cast<uintptr_t>(ws) & 255u) == 0, SD_EWORKSPACE, "gated_linear_bwd: workspace of %zu bytes, need %zu, 256-byte aligned", ws_bytes, need);
    const GatedBwdWs b(M, N, K);
    Workspace w(ws, ws_bytes);
    uint16_t* const dz = static_cast<uint16_t*>(w.take(b.dz));
    float* const sums = static_cast<float*>(w.take(b.sums));
    float* const dx_parts = static_cast<float*>(w.take(b.dx_parts));
    float* const dw_parts = static_cast<float*>(w.take(b.dw_parts));
    const int Np = (2 * N + 7) & ~7;
    const GatedDzCut cut(M, N);
    const int blocks = (int)cut.blocks;
    const bool store = dx || dW;
    if (!SD_DRY_RUN("gated dz%s%s; ", store ? "" : " sums only", dbias ? "" : " no sums")) {
        const dim3 grid((unsigned)(cut.blocks * cut.col_wgs));
        float* const to = blocks == 1 ? dbias : sums;
        auto run = [&](auto* t) {
            using D = std::remove_pointer_t<decltype(t)>;
            const D* const d = static_cast<const D*>(dy);
            auto launch = [&](auto stored, auto summed, auto past) {
                hipLaunchKernelGGL((gated_dz_kernel<D, decltype(stored)::value, decltype(summed)::value, decltype(past)::value>), grid, dim3(GATED_DZ_THREADS), 0, s, d, z, act, dz, to, M, N, Np, cut.rows, blocks);
            };
            const std::true_type yes;
            const std::false_type no;
            const bool past = (int64_t)M * N > 16ll << 20;
            if (!store) launch(no, yes, no);
            else if (dbias && past) launch(yes, yes, yes);
            else if (dbias) launch(yes, yes, no);
            else if (past) launch(yes, no, yes);
            else launch(yes, no, no);
        };
        if (y_dtype == SD_F32) run(static_cast<float*>(nullptr));
        else run(static_cast<__bf16*>(nullptr));
        SD_HIP_CHECK(hipGetLastError());
    }
    if (dbias && blocks > 1) {
        left.sums = sums;
        left.dbias = dbias;
        left.blocks = blocks;
        left.N = 2 * N;
    }
    return launch_products(dz, Np, x, W, dx, dW, dw_dtype, dx_parts, dw_parts, left, M, 2 * N, K, BwdPlan(M, 2 * N, K), s);
}
