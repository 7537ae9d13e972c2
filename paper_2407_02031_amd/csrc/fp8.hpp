// Rows in 8 bits: e4m3 values, K a row, and a scale 2^(s - 127) for each block of 128 of them (the last may be shorter), s a byte.
//
//   amax = max |v| over the block's finite elements;  s the least with amax <= 448 * 2^(s - 127), at least 1;  q = v 2^(127 - s), rounded to
//   nearest, ties to even
//
// A power of two as the scale: v 2^(127 - s) is exact, so an element is rounded once, and the matrix core multiplies by scales itself.  What is not finite becomes NaN and leaves the
// other elements of its block as they are.  s lies between 1 and 247, so neither it nor its inverse is subnormal.
// The scales of a matrix lie block by block, s[block * ld + row], ld a multiple of four: those of the rows of a tile are next to each other.
#pragma once
#include "rows.hpp"

namespace sd {

constexpr int FP8_BLOCK = 128;
inline int fp8_blocks(int K) { return (K + FP8_BLOCK - 1) / FP8_BLOCK; }

// Whether rows in 8 bits can be read or written, and the launch that makes them (rmsnorm.hip)
int fp8_check(const char* who, const char* what, const void* q, const uint8_t* scales, int64_t lds, int64_t rows, int K);
int launch_quantize(const void* x, bool f32, uint8_t* q, uint8_t* scales, int64_t lds, int M, int K, hipStream_t stream);

// |v|, or 0 where v is not finite, as an integer of the same order
__device__ __forceinline__ uint32_t fp8_magnitude(float v) {
    const uint32_t u = __float_as_uint(v) & 0x7fffffffu;
    return u >= 0x7f800000u ? 0u : u;
}
__device__ __forceinline__ uint32_t fp8_magnitude(uint32_t m, f32x4 v) { return max(max(max(m, fp8_magnitude(v[0])), max(fp8_magnitude(v[1]), fp8_magnitude(v[2]))), fp8_magnitude(v[3])); }
// max(m, |v[0]|, ..., |v[3]|), NaN apart: infinite where one of them is
__device__ __forceinline__ float fp8_top(float m, f32x4 v) {
    asm("v_max3_f32 %0, |%1|, |%2|, %0" : "+v"(m) : "v"(v[0]), "v"(v[1]));
    asm("v_max3_f32 %0, |%1|, |%2|, %0" : "+v"(m) : "v"(v[2]), "v"(v[3]));
    return m;
}
// The largest over the 16 lanes of a DPP row, in all of them
__device__ __forceinline__ uint32_t max16(uint32_t m) {
    m = max(m, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)m, 0xB1, 0xf, 0xf, false));
    m = max(m, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)m, 0x4E, 0xf, 0xf, false));
    m = max(m, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)m, 0x141, 0xf, 0xf, false));
    return max(m, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)m, 0x140, 0xf, 0xf, false));
}
// ... over a half of the wavefront, all of whose lanes are there
__device__ __forceinline__ uint32_t max32(uint32_t m) {
    m = max16(m);
    uint32_t a = m, b = m;       // odd rows of a <-> even rows of b
    asm volatile("s_nop 1\n\tv_permlane16_swap_b32 %0, %1" : "+v"(a), "+v"(b));
    return max(a, b);
}
// s of a block's largest magnitude (448 = 1.75 * 2^8), and 2^(127 - s)
__device__ __forceinline__ int fp8_scale(uint32_t amax) { return max(1, (int)((amax + 0x1fffffu) >> 23) - 8); }
__device__ __forceinline__ float fp8_inverse(int s) { return __uint_as_float((uint32_t)(254 - s) << 23); }
// Four elements, times 2^(127 - s), as e4m3 in the order of a row
__device__ __forceinline__ uint32_t fp8_pack(f32x4 v, float inv) {
    // (an infinity is a NaN from here on, whatever the conversion's mode says about overflow)
    auto in = [&](float f) { return fmaf(f, 0.f, f * inv); };
    int w = __builtin_amdgcn_cvt_pk_fp8_f32(in(v[0]), in(v[1]), 0, false);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(in(v[2]), in(v[3]), w, true);
}
// ... of finite ones, or NaN
__device__ __forceinline__ uint32_t fp8_pack_finite(f32x4 v, float inv) {
    int w = __builtin_amdgcn_cvt_pk_fp8_f32(v[0] * inv, v[1] * inv, 0, false);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(v[2] * inv, v[3] * inv, w, true);
}

}  // namespace sd
