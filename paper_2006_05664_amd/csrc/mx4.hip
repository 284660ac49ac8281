// Rows of numbers to microscaled 4 bits (mx4.hpp) and back.  Of every 32 values the largest magnitude's exponent less 2 becomes the factor's, so that it lands in [4, 8); a value over
// the factor is rounded to the nearest E2M1, ties to the even code, 6 at most.  The hardware's conversions round like that.  Bound by memory: a value is read once and
// half a byte written (8192 rows of 4096 in bf16 22.5 us, 3.7 TB/s, waves waiting 84 % of their time: a lane stores four bytes of codes, one in four a byte of
// factors; back 14 us, the codes still in the caches).
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdint>

#include "launch.hpp"
#include "mx4.hpp"
#include "narrow.hpp"
#include "rows.hpp"

namespace {

constexpr int kThreads = 256;
constexpr int kPiece = 8;               // values of a lane: four lanes hold the 32 of a factor

struct Rows4 {
    const void *x;
    long ld_x;
    uint8_t *q, *scale;
    long ld_q, ld_scale;
    long rows;
    int width, tx;
};

// A row's piece, zeros past its end.  Its last values are loaded one by one from places that are there, without a branch each: their latencies overlap.
template <typename T>
__device__ __forceinline__ void load_piece(const T *row, int i, int width, T (&v)[kPiece])
{
    if (i * kPiece + kPiece <= width) __builtin_memcpy(v, row + i * kPiece, sizeof v);
    else {
#pragma unroll
        for (int e = 0; e < kPiece; ++e) v[e] = row[min(i * kPiece + e, width - 1)];
#pragma unroll
        for (int e = 0; e < kPiece; ++e)
            if (i * kPiece + e >= width) v[e] = (T)0.f;
    }
}

template <typename T, int HOLD>
__global__ __launch_bounds__(kThreads)
void quantize_mx4(Rows4 p)
{
    const int tx = p.tx, lane = (int)threadIdx.x & (tx - 1), ty = kThreads >> __builtin_ctz(tx);
    const long row = this_block() * ty + ((int)threadIdx.x >> __builtin_ctz(tx));
    if (row >= p.rows) return;              // all lanes of a row; a factor's four are a row's
    const T *x = (const T *)p.x + row * p.ld_x;
    uint8_t *q = p.q + row * p.ld_q, *scale = p.scale + row * p.ld_scale;
    const int pieces = (p.width + 31) / 32 * (32 / kPiece);
    for (int i0 = lane; i0 < pieces; i0 += tx * HOLD) {
        T v[HOLD][kPiece];
#pragma unroll
        for (int u = 0; u < HOLD; ++u)
            if (i0 + u * tx < pieces) load_piece(x, i0 + u * tx, p.width, v[u]);
#pragma unroll
        for (int u = 0; u < HOLD; ++u) {
            const int i = i0 + u * tx;
            if (i >= pieces) break;
            float f[kPiece];
            unsigned most = 0;              // magnitudes as bits without the sign: in the order of the values, infinities and NaNs last
#pragma unroll
            for (int e = 0; e < kPiece; ++e) {
                f[e] = (float)v[u][e];
                most = max(most, __float_as_uint(f[e]) & 0x7fffffffu);
            }
            most = max(most, (unsigned)__shfl_xor((int)most, 1));
            most = max(most, (unsigned)__shfl_xor((int)most, 2));
            const int exponent = (int)(most >> 23), b = exponent == 255 ? kMx4NaN : max(exponent - 2, 0);
            const float by = mx4_factor(b == kMx4NaN ? 127 : b);
            unsigned w = 0;
            w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, f[0], f[1], by, 0);
            w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, f[2], f[3], by, 1);
            w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, f[4], f[5], by, 2);
            w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, f[6], f[7], by, 3);
            if (b == kMx4NaN) w = 0;
            const int left = (p.width - i * kPiece + 1) / 2;        // bytes of the row from here on
            if (left >= 4) __builtin_memcpy(q + i * 4L, &w, 4);
            else
                for (int o = 0; o < left; ++o) q[i * 4L + o] = (uint8_t)(w >> 8 * o);
            if ((i & 3) == 0) scale[i >> 2] = (uint8_t)b;
        }
    }
}

// The value that a code and its factor stand for, in fp32 where it is exact (6 * 2^127 is an infinity there), rounded once to T.
template <typename T, int HOLD>
__global__ __launch_bounds__(kThreads)
void dequantize_mx4(Rows4 p)
{
    typedef float f32x2 __attribute__((ext_vector_type(2)));
    const int tx = p.tx, lane = (int)threadIdx.x & (tx - 1), ty = kThreads >> __builtin_ctz(tx);
    const long row = this_block() * ty + ((int)threadIdx.x >> __builtin_ctz(tx));
    if (row >= p.rows) return;
    T *x = (T *)p.x + row * p.ld_x;
    const uint8_t *q = p.q + row * p.ld_q, *scale = p.scale + row * p.ld_scale;
    const int pieces = (p.width + kPiece - 1) / kPiece;
    for (int i0 = lane; i0 < pieces; i0 += tx * HOLD) {
        unsigned w[HOLD];
        int b[HOLD];
#pragma unroll
        for (int u = 0; u < HOLD; ++u) {
            const int i = i0 + u * tx, left = (p.width - i * kPiece + 1) / 2;
            w[u] = 0;
            if (i >= pieces) break;
            if (left >= 4) __builtin_memcpy(&w[u], q + i * 4L, 4);
            else
#pragma unroll
                for (int o = 0; o < 3; ++o) w[u] |= (unsigned)q[i * 4L + min(o, left - 1)] << 8 * o;           // what is past the end is not stored
            b[u] = scale[i >> 2];
        }
#pragma unroll
        for (int u = 0; u < HOLD; ++u) {
            const int i = i0 + u * tx;
            if (i >= pieces) break;
            const float by = mx4_factor(b[u] == kMx4NaN ? 127 : b[u]), nan = mx4_factor(kMx4NaN);
            f32x2 f[4] = {__builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w[u], by, 0), __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w[u], by, 1),
                          __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w[u], by, 2), __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w[u], by, 3)};
            T v[kPiece];
#pragma unroll
            for (int e = 0; e < kPiece; ++e) v[e] = narrow<T>(b[u] == kMx4NaN ? nan : f[e / 2][e & 1]);
            if (i * kPiece + kPiece <= p.width) __builtin_memcpy(x + i * kPiece, v, sizeof v);
            else
#pragma unroll
                for (int e = 0; e < kPiece; ++e)
                    if (i * kPiece + e < p.width) x[i * kPiece + e] = v[e];
        }
    }
}

// ------------------------------------------------------------------ host side
using opevo::launch;

// Lanes to a row: a power of two (any multiple of four that leaves fewer idle measures the same at 1062 columns and a fifth more at 7168), and with it how the rows fall into workgroups.
template <typename T>
int run_quantize4(Rows4 p, hipStream_t stream)
{
    const int pieces = (p.width + 31) / 32 * (32 / kPiece);
    p.tx = 4;
    while (p.tx < kThreads && p.tx < pieces) p.tx *= 2;
    const int ty = kThreads / p.tx;
    return launch("quantize_mx4 launch", pieces > p.tx ? quantize_mx4<T, 2> : quantize_mx4<T, 1>, spread((p.rows + ty - 1) / ty), dim3(kThreads), stream, p);
}
template <typename T>
int run_dequantize4(Rows4 p, hipStream_t stream)
{
    const int pieces = (p.width + kPiece - 1) / kPiece;
    p.tx = 1;
    while (p.tx < kThreads && p.tx < pieces) p.tx *= 2;
    const int ty = kThreads / p.tx;
    return launch("dequantize_mx4 launch", pieces > p.tx ? dequantize_mx4<T, 2> : dequantize_mx4<T, 1>, spread((p.rows + ty - 1) / ty), dim3(kThreads), stream, p);
}

int check_rows4(const char *who, const Rows4 &p, int dtype, int64_t rows, int64_t width)
{
    if (!known(dtype)) return fail(OPEVO_E_ARG, "%s: unknown element type %d", who, dtype);
    if (rows < 0 || rows > INT32_MAX) return fail(OPEVO_E_ARG, "%s: %lld rows", who, (long long)rows);
    if (rows == 0) return OPEVO_OK;
    if (int rc = check_rows(who, "x", p.x, p.ld_x, width, size_of(dtype))) return rc;
    if (int rc = check_rows(who, "q", p.q, p.ld_q, (width + 1) / 2, 1)) return rc;
    return check_rows(who, "scale", p.scale, p.ld_scale, (width + 31) / 32, 1);
}

}  // namespace

extern "C" int opevo_quantize_rows_mx4(const void *x, int64_t ld_x, int dtype, int64_t rows, int64_t width, uint8_t *q, int64_t ld_q, uint8_t *scale, int64_t ld_scale, void *stream)
{
    Rows4 p = {x, (long)ld_x, q, scale, (long)ld_q, (long)ld_scale, (long)rows, (int)width, 0};
    if (int rc = check_rows4("quantize_rows_mx4", p, dtype, rows, width)) return rc;
    if (rows == 0) return OPEVO_OK;
    return BY_DTYPE(dtype, run_quantize4, p, static_cast<hipStream_t>(stream));
}

extern "C" int opevo_dequantize_rows_mx4(const uint8_t *q, int64_t ld_q, const uint8_t *scale, int64_t ld_scale, int dtype, int64_t rows, int64_t width, void *x, int64_t ld_x, void *stream)
{
    Rows4 p = {x, (long)ld_x, const_cast<uint8_t *>(q), const_cast<uint8_t *>(scale), (long)ld_q, (long)ld_scale, (long)rows, (int)width, 0};
    if (int rc = check_rows4("dequantize_rows_mx4", p, dtype, rows, width)) return rc;
    if (rows == 0) return OPEVO_OK;
    return BY_DTYPE(dtype, run_dequantize4, p, static_cast<hipStream_t>(stream));
}
