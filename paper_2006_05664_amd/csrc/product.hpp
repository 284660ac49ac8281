// What the products of rows by rows share: finding an expert's rows, operands on their way from memory to registers or the LDS, and stores at any alignment.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

#include "narrow.hpp"

namespace {

typedef int i32x4 __attribute__((ext_vector_type(4)));

// A grid's second extent ends at 65535: tiles of rows go on in the third.
constexpr int kGridY = 65535;
__device__ __forceinline__ long row_tile() { return (long)blockIdx.z * kGridY + blockIdx.y; }

// The rows a workgroup owns, of one expert.
struct Rows { long first, last; int expert; bool zero; };

// Grouped: the tile number `tile` (each expert's rows make whole tiles of BM rows, the last one ragged; after the last expert come the rows that belong
// to none, which get zeros).  Every wave finds it for itself, 64 experts at a time.  Offsets are clamped to the rows there are, so whatever they hold no row
// outside is touched.  False: there is no such tile.
template <typename P>
__device__ __forceinline__ bool find_rows(const P &p, int bm, long tile, Rows *r)
{
    if (!p.offsets) {
        r->first = tile * bm; r->last = p.m; r->expert = 0; r->zero = false;
        return r->first < p.m;
    }
    const int lane = threadIdx.x & 63;
    long seen = 0;
    for (int e0 = 0; e0 <= p.experts; e0 += 64) {
        const int e = e0 + lane;
        long lo = 0, hi = 0;
        if (e <= p.experts) {
            lo = p.offsets[e];
            hi = e < p.experts ? (long)p.offsets[e + 1] : p.m;
            lo = lo < 0 ? 0 : lo > p.m ? p.m : lo;
            hi = hi < lo ? lo : hi > p.m ? p.m : hi;
        }
        const int tiles = (int)((hi - lo + bm - 1) / bm);
        int sum = tiles;
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) {
            const int up = __shfl_up(sum, o);
            if (lane >= o) sum += up;
        }
        const long upto = seen + sum;
        const unsigned long long past = __ballot(upto > tile);
        if (past) {
            const int at = __ffsll(past) - 1;
            const int before = __shfl(sum - tiles, at);
            const int row0 = __shfl((int)lo, at), row1 = __shfl((int)hi, at);
            r->expert = __builtin_amdgcn_readfirstlane(e0 + at);
            r->first = __builtin_amdgcn_readfirstlane(row0) + (tile - seen - __builtin_amdgcn_readfirstlane(before)) * bm;
            r->last = __builtin_amdgcn_readfirstlane(row1);
            r->zero = r->expert == p.experts;
            return true;
        }
        seen += __shfl(sum, 63);
    }
    return false;
}

// Four neighbouring columns of C from `col` on, those that exist.
template <typename T>
__device__ __forceinline__ void store4(T *row, int col, int n, const float (&c)[4])
{
    const T v[4] = {narrow<T>(c[0]), narrow<T>(c[1]), narrow<T>(c[2]), narrow<T>(c[3])};
    if (col + 4 <= n) __builtin_memcpy(row + col, v, sizeof v);
    else
        for (int i = 0; i < 4; ++i)
            if (col + i < n) row[col + i] = v[i];
}

// 16 bytes of a row of K values from k on, zeros past its end.  The piece that K ends in comes as the row's last 16 bytes, shifted.
__device__ __forceinline__ i32x4 load_chunk(const int8_t *row, int k, int end)
{
    i32x4 v = {0, 0, 0, 0};
    if (k + 16 <= end) __builtin_memcpy(&v, row + k, 16);
    else if (k < end) {
        if (end >= 16) {
            unsigned __int128 w;
            __builtin_memcpy(&w, row + end - 16, 16);
            w >>= 8 * (k + 16 - end);
            __builtin_memcpy(&v, &w, 16);
        } else {
            for (int i = 0; k + i < end; ++i) v[i >> 2] |= (int)(uint8_t)row[k + i] << (8 * (i & 3));
        }
    }
    return v;
}

// lane i's 16 bytes from base + off to LDS at lds + 16 i; the kernel places every wait these loads need itself.  The base goes through a scalar copy: a
// vector instruction that wrote it (a lane brought back into a scalar register) is followed by wait states only where the compiler sees a memory instruction.
__device__ __forceinline__ void load_to_lds(const int8_t *base, unsigned off, unsigned lds)
{
    const int8_t *copy;
    asm volatile("s_mov_b32 m0, %3\n\ts_mov_b64 %0, %2\n\tglobal_load_lds_dwordx4 %1, %0" : "=&s"(copy) : "v"(off), "s"(base), "s"(lds) : "memory", "m0");
}
#define WAIT_LGKM_VMCNT(n) __builtin_amdgcn_s_waitcnt(((n) & 0xf) | (((n) >> 4) << 14) | (0x7 << 4))
#define WAIT_LGKM() __builtin_amdgcn_s_waitcnt(0xf | (0x3 << 14) | (0x7 << 4))
#define BARRIER() do { asm volatile("" ::: "memory"); __builtin_amdgcn_s_barrier(); asm volatile("" ::: "memory"); } while (0)

__device__ __forceinline__ int uniform(int v) { return __builtin_amdgcn_readfirstlane(v); }
__device__ __forceinline__ const int8_t *uniform(const int8_t *p)
{
    const unsigned long long v = (unsigned long long)p;
    return (const int8_t *)(((unsigned long long)(unsigned)uniform((int)(v >> 32)) << 32) | (unsigned)uniform((int)v));
}

}  // namespace
