// Microscaled 4-bit numbers: E2M1 values (0, 0.5, 1, 1.5, 2, 3, 4, 6 and their negatives), two a byte with the earlier one in the low half, and for every 32
// of a row a byte b that stands for the factor 2^(b - 127), or for NaN where it is 255.
#pragma once

#include <hip/hip_runtime.h>

namespace {

constexpr int kMx4NaN = 255;

// The factor in fp32.  2^-127 is subnormal there; the conversions take it.
__device__ __forceinline__ float mx4_factor(int b) { return __uint_as_float(b == kMx4NaN ? 0x7fc00000u : b == 0 ? 0x00400000u : (unsigned)b << 23); }

}  // namespace
