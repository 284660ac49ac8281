// Microscaled 4-bit numbers: E2M1 values (0, 0.5, 1, 1.5, 2, 3, 4, 6 and their negatives), two a byte with the earlier one in the low half, and for every 32
// of a row a byte b that stands for the factor 2^(b - 127), or for NaN where it is 255.
#pragma once

#include <hip/hip_runtime.h>

#include "product.hpp"

namespace {

constexpr int kMx4NaN = 255;

// The factor in fp32.  2^-127 is subnormal there; the conversions take it.
__device__ __forceinline__ float mx4_factor(int b) { return __uint_as_float(b == kMx4NaN ? 0x7fc00000u : b == 0 ? 0x00400000u : (unsigned)b << 23); }

// Codes from byte k of a row on that ends at byte `end`, the last one of which has half a byte too many where `odd`.
__device__ __forceinline__ i32x4 without_half_byte(i32x4 v, int k, int end, bool odd)
{
    const int last = end - 1 - k;
    if (odd && last >= 0 && last < 16)
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (last >> 2 == i) v[i] &= ~(0xf0 << 8 * (last & 3));
    return v;
}
// 16 bytes of a row from byte k on, a multiple of 16, zeros past its end (and in the half byte past an odd K).  LONG: of a row of 16 bytes or more, without a branch, so that the latencies of
// several overlap: the piece that the row ends in comes as its last 16 bytes, shifted.
template <bool LONG> __device__ __forceinline__ i32x4 load_codes(const uint8_t *row, int k, int end, bool odd)
{
    if (!LONG) return without_half_byte(load_chunk((const int8_t *)row, k, end), k, end, odd);
    i32x4 v, w;
    __builtin_memcpy(&v, row + min(k, end - 16), 16);
    const int by = (16 - end % 16) % 16;                    // alike for all lanes
    w = by & 8 ? i32x4{v[2], v[3], 0, 0} : v;
    w = by & 4 ? i32x4{w[1], w[2], w[3], 0} : w;
    w = i32x4{(int)__builtin_amdgcn_alignbyte(w[1], w[0], by), (int)__builtin_amdgcn_alignbyte(w[2], w[1], by), (int)__builtin_amdgcn_alignbyte(w[3], w[2], by), (int)__builtin_amdgcn_alignbyte(0, w[3], by)};
    w = k < end ? w : i32x4{0, 0, 0, 0};
    return without_half_byte(k + 16 <= end ? v : w, k, end, odd);
}
// Four factors of a row from block b on, zeros past its end: with codes of zero any factor but NaN gives zero.  LONG: of a row of four or more, without a branch.
template <bool LONG> __device__ __forceinline__ int load_factors(const uint8_t *row, int b, int blocks)
{
    unsigned v = 0;
    if (LONG) {
        const int at = min(b, blocks - 4);
        __builtin_memcpy(&v, row + at, 4);
        return b - at >= 4 ? 0 : (int)(v >> 8 * (b - at));
    }
    if (b + 4 <= blocks) __builtin_memcpy(&v, row + b, 4);
    else
        for (int i = 0; b + i < blocks; ++i) v |= (unsigned)row[b + i] << 8 * i;
    return (int)v;
}

}  // namespace
