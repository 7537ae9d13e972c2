// Rows that a norm holds in registers: how the threads of a row share it, their sums, and which kernel a row length takes (layernorm.hip, rmsnorm.hip).
#pragma once
#include "rows.hpp"

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

// Threads a row and chunks a thread, from the row's length: a wavefront up to 2048 elements, 256 threads up to 8192, and 16 threads for short rows, of which a wavefront's
// lanes would have little each (us, 64 / 16 threads a row: 32768 rows forward of 64 10.7 / 4.8, of 128 11.8 / 8.2, of 320 19.3 / 14.1; backward with gradients of the weights of 64 15.3 / 9.6, of 128
// 17.0 / 14.4, but of 256 19.7 / 25.3, 320 25.8 / 27.8: a thread's sums of columns take the registers of the wavefronts that would hide its loads).
template <int TPR_, int J_, int JW_>
struct LnShape { static constexpr int TPR = TPR_, J = J_, JW = JW_; };
template <bool BACKWARD, class F>
int ln_by_length(int C, F f) {
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
inline int ln_threads_per_row(int C, bool backward) { return C <= (backward ? 128 : 512) ? 16 : C <= 2048 ? 64 : C <= 8192 ? 256 : 1024; }
template <class F>
int by_type(int dtype, F f) {
    if (dtype == SD_F32) return f(static_cast<float*>(nullptr));
    return f(static_cast<__bf16*>(nullptr));
}

}  // namespace sd
