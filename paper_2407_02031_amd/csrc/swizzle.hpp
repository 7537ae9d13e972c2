// Where a chunk of a row lies in LDS: a function of whole numbers alone, for the kernels and for programs on the CPU that go through what they do.
#pragma once
#ifdef __HIPCC__
#define SD_INDEX_FN __host__ __device__ __forceinline__
#else
#define SD_INDEX_FN inline
#endif

namespace sd {

// XOR swizzle of the 16-byte chunk index inside an LDS row of CPR chunks (8: 128-byte rows,
// 4: 64-byte rows): any 16 consecutive rows put the same logical chunk in 16 distinct
// 16-byte slots of a 256-byte bank window.
template <int CPR>
SD_INDEX_FN constexpr int swz(int row, int chunk) {
    return CPR == 8 ? (chunk ^ ((row >> 1) & 7)) : (chunk ^ ((row >> 2) & 3));
}

}  // namespace sd
