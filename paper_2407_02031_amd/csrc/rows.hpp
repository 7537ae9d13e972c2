// Four neighbouring elements of a row, fp32 or bf16, as fp32: what the row operators (layer norm, the slope of an
// activation, column sums) read and write.  Rows of any length: an access need only be aligned to one element, which the
// hardware allows for global memory, so rows of odd length take the same wide accesses as others.
#pragma once
#include "common.hpp"

namespace sd {

typedef float f32x4u __attribute__((ext_vector_type(4), aligned(4)));
typedef __bf16 bf16x4u __attribute__((ext_vector_type(4), aligned(2)));

__device__ __forceinline__ f32x4 load4(const float* p) { return *reinterpret_cast<const f32x4u*>(p); }
__device__ __forceinline__ f32x4 load4(const __bf16* p) {
    const bf16x4u v = *reinterpret_cast<const bf16x4u*>(p);
    return f32x4{(float)v[0], (float)v[1], (float)v[2], (float)v[3]};
}
__device__ __forceinline__ void store4(float* p, f32x4 v) { *reinterpret_cast<f32x4u*>(p) = v; }
__device__ __forceinline__ void store4(__bf16* p, f32x4 v) {
    *reinterpret_cast<bf16x4u*>(p) = bf16x4u{(__bf16)v[0], (__bf16)v[1], (__bf16)v[2], (__bf16)v[3]};
}
// eight of them
struct f32x8 { f32x4 lo, hi; };
typedef __bf16 bf16x8u __attribute__((ext_vector_type(8), aligned(2)));
__device__ __forceinline__ f32x8 load8(const float* p) { return f32x8{load4(p), load4(p + 4)}; }
__device__ __forceinline__ f32x8 load8(const __bf16* p) {
    const bf16x8u v = *reinterpret_cast<const bf16x8u*>(p);
    return f32x8{f32x4{(float)v[0], (float)v[1], (float)v[2], (float)v[3]}, f32x4{(float)v[4], (float)v[5], (float)v[6], (float)v[7]}};
}
__device__ __forceinline__ void store8(__bf16* p, const f32x8& v) {
    *reinterpret_cast<bf16x8u*>(p) =
        bf16x8u{(__bf16)v.lo[0], (__bf16)v.lo[1], (__bf16)v.lo[2], (__bf16)v.lo[3], (__bf16)v.hi[0], (__bf16)v.hi[1], (__bf16)v.hi[2], (__bf16)v.hi[3]};
}

// out0[c] = sum over g of partials[g][c], c < n0, and out1[c - n0] for n0 <= c < n0 + n1; rows of `partials` are n0 + n1
// long.  In a fixed order.  An output that is null is not written.
int launch_sum_partials(const float* partials, int G, float* out0, int n0, float* out1, int n1, hipStream_t stream);

}  // namespace sd
