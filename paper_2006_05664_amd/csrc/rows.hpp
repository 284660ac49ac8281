// Rows of elements on the device: pieces, grids of as many workgroups as there are rows, and the checks of a caller's rows.
#pragma once

#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdint>

#include "launch.hpp"

namespace {

// A launch has fewer than 2^32 threads along an extent of its grid: workgroups go on in the third after as many as make 2^31.
__device__ __forceinline__ long this_block() { return (long)blockIdx.z * gridDim.x + blockIdx.x; }
inline dim3 spread(int64_t blocks, int64_t parts = 1, int threads = 256)
{
    const int64_t most = ((int64_t)1 << 31) / threads;
    return dim3((unsigned)std::min(blocks, most), (unsigned)parts, (unsigned)((blocks + most - 1) / most));
}

// 16 bytes of a row.
template <typename T> struct Vec {
    static constexpr int n = 16 / sizeof(T);
    T v[n];
};

// Stores 16 bytes that no kernel before the end of this one reads: they leave for memory at once, where lines left in the L2s are written back at the end of the launch.
// Every address takes them.
__device__ __forceinline__ void store_away(void *to, const void *from)
{
    typedef int any __attribute__((ext_vector_type(4), aligned(1)));
    any v;
    __builtin_memcpy(&v, from, 16);
    __builtin_nontemporal_store(v, static_cast<any *>(to));
}

using opevo::fail;

inline bool aligned(const void *p, size_t to) { return reinterpret_cast<uintptr_t>(p) % to == 0; }
inline size_t size_of(int dtype) { return dtype == OPEVO_F32 ? 4 : 2; }
inline bool known(int dtype) { return dtype == OPEVO_F32 || dtype == OPEVO_BF16 || dtype == OPEVO_F16; }

// rows of `width` elements, `ld` apart
inline int check_rows(const char *who, const char *name, const void *p, int64_t ld, int64_t width, size_t bytes)
{
    if (!p) return fail(OPEVO_E_ARG, "%s: %s is NULL", who, name);
    if (!aligned(p, bytes)) return fail(OPEVO_E_ARG, "%s: %s is not aligned to its elements", who, name);
    if (width < 1 || width > (1 << 24)) return fail(OPEVO_E_ARG, "%s: rows of %lld elements (1 to 2^24)", who, (long long)width);
    if (ld < width || ld > ((int64_t)1 << 40)) return fail(OPEVO_E_ARG, "%s: rows of %s are %lld apart, shorter than their %lld elements or beyond 2^40", who, name, (long long)ld, (long long)width);
    return OPEVO_OK;
}
inline int check_words(const char *who, const char *name, const void *p)
{
    return p && aligned(p, 4) ? OPEVO_OK : fail(OPEVO_E_ARG, "%s: %s is NULL or not aligned to 4 bytes", who, name);
}

}  // namespace

#define BY_DTYPE(dtype, call, ...)                                          \
    ((dtype) == OPEVO_F32 ? call<float>(__VA_ARGS__)                        \
     : (dtype) == OPEVO_BF16 ? call<__bf16>(__VA_ARGS__) : call<_Float16>(__VA_ARGS__))
