// Products of 8-bit integers with a scale for each row of either operand:
//   C[m, n] = (sum_k A[m, k] B[n, k]) * (sa[m] * sb[n]),
// the sum in 32-bit integers, exactly (K < 2^17, so that 128 * 128 * K fits), one rounding of it to fp32, one for each product, and one to
// the output type.  B holds an output channel a row, as the weights of a layer are stored, so both operands are read along K.  The grouped form gives each
// range of rows offsets[e] .. offsets[e + 1] a B of its own; the offsets are known on the device only.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdint>

#include "kernel.hpp"
#include "narrow.hpp"

namespace {

typedef int i32x4 __attribute__((ext_vector_type(4)));

// What one call computes.  Plain: experts = 0, offsets = NULL.  Grouped: B has experts * N rows.
struct Product {
    const int8_t *a, *b;
    long lda, ldb;
    const float *sa, *sb;
    const int *offsets;
    int experts;
    void *c;
    long ldc;
    int out;            // opevo_dtype
    long m;
    int n, k;
};

// The rows a workgroup owns, of one expert.
struct Rows { long first, last; int expert; bool zero; };

// Grouped: the tile number `tile` (each expert's rows make whole tiles of BM rows, the last one ragged; after the last expert come the rows that belong
// to none, which get zeros).  Every wave finds it for itself, 64 experts at a time.  Offsets are clamped to the rows there are, so whatever they hold no row
// outside is touched.  False: there is no such tile.
__device__ __forceinline__ bool find_rows(const Product &p, int bm, long tile, Rows *r)
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
__device__ __forceinline__ void store4(T *row, int col, int n, float a, float b, float c, float d)
{
    const T v[4] = {narrow<T>(a), narrow<T>(b), narrow<T>(c), narrow<T>(d)};
    if (col + 4 <= n) __builtin_memcpy(row + col, v, sizeof v);
    else
        for (int i = 0; i < 4; ++i)
            if (col + i < n) row[col + i] = v[i];
}

// 16 bytes of a row of K values from k on, zeros past its end.
__device__ __forceinline__ i32x4 load_chunk(const int8_t *row, int k, int end)
{
    i32x4 v = {0, 0, 0, 0};
    if (k + 16 <= end) __builtin_memcpy(&v, row + k, 16);
    else if (k < end) {
        for (int i = 0; k + i < end; ++i) v[i >> 2] |= (int)(uint8_t)row[k + i] << (8 * (i & 3));
    }
    return v;
}

// Any extents, any alignment.  A workgroup of four waves owns 64 x 64; slabs of 64 values go through registers into LDS, rows 16 bytes apart
// from a multiple of the banks.  The MFMA takes B's rows as its first operand, so that a lane holds four neighbouring columns of one row of C.
template <typename T>
__global__ __launch_bounds__(256)
void product_any(Product p)
{
    constexpr int BM = 64, BN = 64, BK = 64, PITCH = BK + 16;
    __shared__ __attribute__((aligned(16))) int8_t As[BM * PITCH], Bs[BN * PITCH];
    Rows r;
    if (!find_rows(p, BM, blockIdx.y, &r)) return;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, wm = wave >> 1, wn = wave & 1;
    const int n0 = blockIdx.x * BN;
    i32x4 acc[2][2] = {};
    if (!r.zero) {
        const int row = tid >> 2, kc = (tid & 3) * 16;
        const long am = r.first + row < r.last ? r.first + row : r.last - 1;
        const int bn = n0 + row < p.n ? n0 + row : p.n - 1;
        const int8_t *arow = p.a + am * p.lda, *brow = p.b + ((long)r.expert * p.n + bn) * p.ldb;
        for (int k0 = 0; k0 < p.k; k0 += BK) {
            const i32x4 av = load_chunk(arow, k0 + kc, p.k), bv = load_chunk(brow, k0 + kc, p.k);
            __syncthreads();
            *(i32x4 *)(As + row * PITCH + kc) = av;
            *(i32x4 *)(Bs + row * PITCH + kc) = bv;
            __syncthreads();
            i32x4 af[2], bf[2];
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                af[i] = *(const i32x4 *)(As + (wm * 32 + i * 16 + (lane & 15)) * PITCH + (lane >> 4) * 16);
                bf[i] = *(const i32x4 *)(Bs + (wn * 32 + i * 16 + (lane & 15)) * PITCH + (lane >> 4) * 16);
            }
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int j = 0; j < 2; ++j) acc[i][j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(bf[j], af[i], acc[i][j], 0, 0, 0);
        }
    }
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const long m = r.first + wm * 32 + i * 16 + (lane & 15);
        if (m >= r.last) continue;
        const float sa = r.zero ? 0.f : p.sa[m];
        T *row = (T *)p.c + m * p.ldc;
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const int col = n0 + wn * 32 + j * 16 + (lane >> 4) * 4;
            float v[4];
#pragma unroll
            for (int e = 0; e < 4; ++e)
                v[e] = !r.zero && col + e < p.n ? (float)acc[i][j][e] * (sa * p.sb[(long)r.expert * p.n + col + e]) : 0.f;
            store4(row, col, p.n, v[0], v[1], v[2], v[3]);
        }
    }
}

using opevo::fail;

template <typename T>
int run_product(const Product &p, hipStream_t stream)
{
    // grouped: an expert's last tile is ragged, and so is that of the rows of none
    const int64_t tiles = p.offsets ? std::min<int64_t>(p.m, p.m / 64 + p.experts + 1) : (p.m + 63) / 64;
    hipLaunchKernelGGL(product_any<T>, dim3((unsigned)((p.n + 63) / 64), (unsigned)tiles), dim3(256), 0, stream, p);
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? OPEVO_OK : opevo::hip_fail(e, "product launch");
}

int check_operand(const char *who, const char *name, const void *p, int64_t ld, int64_t width, size_t bytes)
{
    if (!p || reinterpret_cast<uintptr_t>(p) % bytes) return fail(OPEVO_E_ARG, "%s: %s is NULL or not aligned to its elements", who, name);
    if (ld < width || ld > ((int64_t)1 << 40)) return fail(OPEVO_E_ARG, "%s: rows of %s are %lld apart, shorter than their %lld elements or beyond 2^40", who, name, (long long)ld, (long long)width);
    return OPEVO_OK;
}

int product(const char *who, Product &p, int64_t m, int64_t n, int64_t k, int experts, void *stream)
{
    if (p.out != OPEVO_F32 && p.out != OPEVO_BF16 && p.out != OPEVO_F16) return fail(OPEVO_E_ARG, "%s: unknown output type %d", who, p.out);
    if (m < 0 || n < 0 || m > (1 << 21) || n > (1 << 24)) return fail(OPEVO_E_ARG, "%s: %lld rows (at most 2^21) and %lld columns (at most 2^24)", who, (long long)m, (long long)n);
    if (k < 1 || k >= (1 << 17)) return fail(OPEVO_E_ARG, "%s: K = %lld (1 to 2^17 - 1, so that the sum fits 32 bits)", who, (long long)k);
    if (m == 0 || n == 0) return OPEVO_OK;
    if (int rc = check_operand(who, "a", p.a, p.lda, k, 1)) return rc;
    if (int rc = check_operand(who, "b", p.b, p.ldb, k, 1)) return rc;
    if (int rc = check_operand(who, "c", p.c, p.ldc, n, p.out == OPEVO_F32 ? 4 : 2)) return rc;
    if (int rc = check_operand(who, "scale_a", p.sa, 1, 1, 4)) return rc;
    if (int rc = check_operand(who, "scale_b", p.sb, 1, 1, 4)) return rc;
    p.m = m; p.n = (int)n; p.k = (int)k; p.experts = experts;
    const hipStream_t on = static_cast<hipStream_t>(stream);
    return p.out == OPEVO_F32 ? run_product<float>(p, on) : p.out == OPEVO_BF16 ? run_product<__bf16>(p, on) : run_product<_Float16>(p, on);
}

}  // namespace

extern "C" int opevo_matmul_i8(const int8_t *a, int64_t lda, const float *scale_a, const int8_t *b, int64_t ldb, const float *scale_b, void *c, int64_t ldc,
                               int out_dtype, int64_t M, int64_t N, int64_t K, void *stream)
{
    Product p = {a, b, (long)lda, (long)ldb, scale_a, scale_b, nullptr, 0, c, (long)ldc, out_dtype, 0, 0, 0};
    return product("matmul_i8", p, M, N, K, 0, stream);
}

extern "C" int opevo_matmul_i8_grouped(const int8_t *a, int64_t lda, const float *scale_a, const int8_t *b, int64_t ldb, const float *scale_b,
                                       const int32_t *offsets, int experts, void *c, int64_t ldc, int out_dtype, int64_t rows, int64_t N, int64_t K,
                                       void *stream)
{
    const char *who = "matmul_i8_grouped";
    if (experts < 1 || experts > OPEVO_ROUTE_MAX_EXPERTS) return fail(OPEVO_E_ARG, "%s: %d experts (1 to %d)", who, experts, OPEVO_ROUTE_MAX_EXPERTS);
    if (rows > 0 && N > 0 && (!offsets || reinterpret_cast<uintptr_t>(offsets) % 4)) return fail(OPEVO_E_ARG, "%s: offsets is NULL or not aligned to 4 bytes", who);
    Product p = {a, b, (long)lda, (long)ldb, scale_a, scale_b, offsets, experts, c, (long)ldc, out_dtype, 0, 0, 0};
    return product(who, p, rows, N, K, experts, stream);
}
