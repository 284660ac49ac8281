// RMS norm of rows with the residual's addition in front of it, its rows in 8 bits, and its gradient:
//   s = round(x + r),  i = 1 / sqrt(mean(s^2) + eps),  y = s i w,
//   dx = i (w dy - s i^2 mean(w dy s)) + ds,  dw = sum over rows of dy s i.
// Bound by memory: a row is read once, held in registers while its sum of squares is formed, and written from there.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cfloat>
#include <cstdint>
#include <type_traits>

#include "launch.hpp"
#include "narrow.hpp"
#include "rows.hpp"

namespace {

constexpr int kThreads = 256;           // of a workgroup; as many as a row's lanes where those are more
constexpr int kMostLanes = 512;

// How a row falls into pieces of 16 bytes.  kWhole: without a rest.  kOverlap: the last piece ends with the row and shares elements with the one before it; both write the same values, after
// all pieces of the row have been read (a sum may stand in the place of an input), so the row has to be held in registers.  kRest: the last piece is taken element by element, which
// makes branches of every access (32 rows of 4096 bf16: 4.2 us instead of 3.4).
enum Way { kWhole, kOverlap, kRest };
template <typename T, Way WAY> struct Row {
    static constexpr int n = Vec<T>::n;
    int width, count;
    __device__ explicit Row(int w) : width(w), count((w + n - 1) / n) {}
    __device__ __forceinline__ int first(int i) const { return WAY == kOverlap ? min(i * n, width - n) : i * n; }
    // how many of its elements the piece before has too
    __device__ __forceinline__ int twice(int i) const { return WAY == kOverlap ? i * n - first(i) : 0; }
    __device__ __forceinline__ Vec<T> load(const T *row, int i) const
    {
        Vec<T> v = {};
        if (WAY != kRest || i * n + n <= width) __builtin_memcpy(&v, row + first(i), 16);
        else
#pragma unroll
            for (int e = 0; e < n; ++e)
                if (i * n + e < width) v.v[e] = row[i * n + e];
        return v;
    }
    template <typename O> __device__ __forceinline__ void store(O *row, int i, const O (&v)[n]) const
    {
        if (WAY != kRest || i * n + n <= width) {
            // 16 bytes past the L2s: 8192 rows of 4096 bf16 37.8 -> 35.7 us, 1024 of them 6.4 -> 5.3, with a kernel that reads them next 48.7 -> 47.0 and 10.3 -> 9.1.  Not the 8 of 8-bit rows
            // (16384 of 4096 and a reader: 93 -> 96).
            if (sizeof v == 16) store_away(row + first(i), v);
            else __builtin_memcpy(row + first(i), v, sizeof v);
        }
        else
#pragma unroll
            for (int e = 0; e < n; ++e)
                if (i * n + e < width) row[i * n + e] = v[e];
    }
};

// Lanes of a row: `tx` side by side, a power of two.  What they hold is combined in an order that depends on tx alone.
template <typename V, typename F> __device__ __forceinline__ V of_wave(V v, int tx, F &&f)
{
    for (int o = 1; o < tx && o < 64; o <<= 1) v = f(v, (V)__shfl_xor(v, o));
    return v;
}
template <typename V, typename F> __device__ __forceinline__ V of_waves(const V *red, int tx, F &&f)
{
    const int w0 = (int)((threadIdx.x >> __builtin_ctz(tx)) << (__builtin_ctz(tx) - 6));
    V v = red[w0];
    for (int w = 1; w < tx / 64; ++w) v = f(v, red[w0 + w]);
    return v;
}

// s w as the quantiser takes it: without rounding.  The product of two bf16 has 16 bits and that of two fp16 22, so fp32 holds it; fp32's takes 48 and goes into fp64.  Products of two bf16 below 2^-126 lose
// bits in fp32, but what is less than a 256th of the row's largest is 0 in 8 bits: rows whose largest is below kTiny, and they alone, are taken once more, in fp64.
template <typename T> struct Exact { typedef float type; };
template <> struct Exact<float> { typedef double type; };
constexpr float kTiny = 0x1p-110f;

// q = round(127 v / a).  v times 127 / a in fp32 is off by at most three roundings, 127 * 3 * 2^-24 = 2.3e-5, and rounds to the same integer unless it is within 4e-5 of
// the middle between two; then the quotients of the piece are formed in fp64, where the middle is hit only by quotients that are there.
template <typename V> struct RowTo8 {
    V a, pre;
    float inv;
    bool on;
    __device__ explicit RowTo8(V a_) : a(a_)
    {
        pre = a > (V)1e30 ? (V)0x1p-96 : a < (V)1e-30 ? (V)0x1p96 : (V)1;   // neither the factor nor its product overflows
        if constexpr (sizeof(V) == 8)
            if (a < 1e-60) pre = 0x1p192;           // products of two fp32 go down to 2^-298
        inv = 127.f / (float)(a * pre);
        on = a > 0 && a <= (V)FLT_MAX;
    }
    template <int N> __device__ __forceinline__ void operator()(const V (&v)[N], int8_t (&q)[N]) const
    {
        constexpr float kRound = 12582912.f;                // 1.5 * 2^23: what is added to it is rounded to an integer, in its low bits
        float off = 0.f;
#pragma unroll
        for (int e = 0; e < N; ++e) {
            const float f = (float)(v[e] * pre), r = fmaf(f, inv, kRound);
            off = fmaxf(off, fabsf(fmaf(f, inv, kRound - r)));
            q[e] = (int8_t)(on ? (int)(__float_as_uint(r) & 0xff) : 0);
        }
        if (on && off > 0.49996f)
#pragma unroll 1
            for (int e = 0; e < N; ++e) q[e] = (int8_t)(int)rint(127.0 * (double)v[e] / (double)a);
    }
};

struct Norm {
    const void *x, *residual, *weight;
    long ld_x, ld_residual;
    void *sum;
    long ld_sum;
    void *y;                // the norm in the rows' type, or in 8 bits
    long ld_y;
    float *per_row;         // 1 / rms, or the scale of a row in 8 bits; may be NULL in the first case
    long rows;
    int width, tx;
    float eps;
};

// 16384 rows of 4096 bf16 with a residual: 537 MB in 87 us (6.2 TB/s; a large copy takes 104 for as many bytes); in 8 bits 96, with more instructions a value than memory hides.  32 rows: 3.2 us, a launch and a
// chain of latencies.  As many lanes as a row has pieces, up to 512: two pieces on 256 lanes and four on 128 take as long, eight on 64 half as long again.
template <typename T, int HOLD, bool TO8, Way WAY>
__global__ __launch_bounds__(kMostLanes)
void norm_rows(Norm p)
{
    typedef typename Exact<T>::type V;
    constexpr int n = Vec<T>::n;
    __shared__ float red[kMostLanes / 64];
    __shared__ V red8[kMostLanes / 64];
    const int tx = p.tx, lane = (int)threadIdx.x & (tx - 1);
    const long row = this_block() * (blockDim.x >> __builtin_ctz(tx)) + (threadIdx.x >> __builtin_ctz(tx));
    const bool on = row < p.rows;
    const Row<T, WAY> at(p.width);
    const int count = on ? at.count : 0;
    const T *x = (const T *)p.x + row * p.ld_x, *r = (const T *)p.residual + row * p.ld_residual, *w = (const T *)p.weight;
    auto summed = [&](const Vec<T> &x, const Vec<T> &r) {
        Vec<T> s;
#pragma unroll
        for (int e = 0; e < n; ++e) s.v[e] = narrow<T>((float)x.v[e] + (float)r.v[e]);
        return s;
    };
    auto weights = [&](int i) {
        if (w) return at.load(w, i);
        Vec<T> one;
#pragma unroll
        for (int e = 0; e < n; ++e) one.v[e] = (T)1.f;
        return one;
    };
    Vec<T> s[HOLD], by[HOLD];
#pragma unroll
    for (int u = 0; u < HOLD; ++u)
        if (lane + u * tx < count) s[u] = at.load(x, lane + u * tx);
    if (p.residual) {
        Vec<T> add[HOLD];
#pragma unroll
        for (int u = 0; u < HOLD; ++u)
            if (lane + u * tx < count) add[u] = at.load(r, lane + u * tx);
#pragma unroll
        for (int u = 0; u < HOLD; ++u)
            if (lane + u * tx < count) by[u] = weights(lane + u * tx);
#pragma unroll
        for (int u = 0; u < HOLD; ++u)
            if (lane + u * tx < count) s[u] = summed(s[u], add[u]);
    } else {
#pragma unroll
        for (int u = 0; u < HOLD; ++u)
            if (lane + u * tx < count) by[u] = weights(lane + u * tx);
    }
    float squares = 0.f;
    V most = 0;
    auto look = [&](int twice, const Vec<T> &v, const Vec<T> &by) {
#pragma unroll
        for (int e = 0; e < n; ++e)
            if (e >= twice) squares = fmaf((float)v.v[e], (float)v.v[e], squares);
        if (TO8) {
#pragma unroll
            for (int e = 0; e < n; ++e) {
                V m = fabs((V)v.v[e] * (V)by.v[e]);
                if (!(m <= (V)FLT_MAX)) m = (V)INFINITY;    // NaN too: a maximum passes over it
                most = fmax(most, m);
            }
        }
    };
#pragma unroll
    for (int u = 0; u < HOLD; ++u)
        if (lane + u * tx < count) look(at.twice(lane + u * tx), s[u], by[u]);
    // pieces that no lane holds are read, and added up, once more when they are written
    auto again = [&](int i) { return p.residual ? summed(at.load(x, i), at.load(r, i)) : at.load(x, i); };
    if (WAY != kOverlap)
        for (int i = lane + HOLD * tx; i < count; i += tx) look(0, again(i), weights(i));
    const auto add = [](float a, float b) { return a + b; };
    const auto larger = [](V a, V b) { return fmax(a, b); };
    squares = of_wave(squares, tx, add);
    if (TO8) most = of_wave(most, tx, larger);
    if (tx > 64) {                          // alike for the whole workgroup
        if ((threadIdx.x & 63) == 0) {
            red[threadIdx.x >> 6] = squares;
            if (TO8) red8[threadIdx.x >> 6] = most;
        }
        __syncthreads();
        squares = of_waves(red, tx, add);
        if (TO8) most = of_waves(red8, tx, larger);
    }
    const float inv = 1.f / sqrtf(squares / (float)p.width + p.eps);
    constexpr bool TWICE = TO8 && std::is_same<T, __bf16>::value;      // rows may be taken once more, by waves that meet
    if (!TWICE && !on) return;          // (8192 rows of 4096 fp32 in 8 bits 69 us, 73 without)
    const RowTo8<V> to8(most);
    T *sum = (T *)p.sum + row * p.ld_sum;
    auto write = [&](int i, const Vec<T> &v, const Vec<T> &by) {
        if (p.sum) at.store(sum, i, v.v);
        if constexpr (TO8) {
            V product[n];
            int8_t q[n];
#pragma unroll
            for (int e = 0; e < n; ++e) product[e] = (V)v.v[e] * (V)by.v[e];
            to8(product, q);
            at.store((int8_t *)p.y + row * p.ld_y, i, q);
        } else {
            Vec<T> y;
#pragma unroll
            for (int e = 0; e < n; ++e) y.v[e] = narrow<T>((float)v.v[e] * inv * (float)by.v[e]);
            at.store((T *)p.y + row * p.ld_y, i, y.v);
        }
    };
#pragma unroll
    for (int u = 0; u < HOLD; ++u)
        if (lane + u * tx < count) write(lane + u * tx, s[u], by[u]);
    if (WAY != kOverlap)
        for (int i = lane + HOLD * tx; i < count; i += tx) write(i, again(i), weights(i));
    const auto scale = [&](auto most) { return most <= FLT_MAX ? (float)((double)most * (double)inv / 127.0) : __uint_as_float(0x7fc00000u); };      // in fp64: a i may be beyond fp32 and its 127th part not
    if (on && lane == 0 && p.per_row) p.per_row[row] = TO8 ? scale(most) : inv;
    if constexpr (TWICE) {
        // Behind what all rows take, where it costs them least (16384 rows of 4096: 97 us without, 100 like this, 101 - 103 with it in front); s stands in memory by now, and a lane reads what it
        // has written.
        bool tiny = on && most < kTiny;
        if (tx == 128) {                    // alike for the whole workgroup, whose waves meet: two rows
            const int other = ((int)threadIdx.x >> 6 & ~1) ^ 2;
            tiny |= (row ^ 1) < p.rows && fmaxf(red8[other], red8[other + 1]) < kTiny;
        }
        if (__ballot(tiny) == 0) return;
        __shared__ double red64[kMostLanes / 64];
        const T *from = p.sum ? sum : x;
        double largest = 0;
        auto each = [&](auto &&f) {
#pragma unroll 1
            for (int i = lane; i < count; i += tx)
#pragma unroll 1
                for (int c = at.first(i); c < min(at.first(i) + n, p.width); ++c) {
                    T s;
                    __builtin_memcpy(&s, from + c, sizeof s);           // may be what was stored there as another type
                    f(c, w ? (double)s * (double)w[c] : (double)s);
                }
        };
        each([&](int, double v) { largest = fmax(largest, fabs(v) <= (double)FLT_MAX ? fabs(v) : (double)INFINITY); });
        const auto larger64 = [](double a, double b) { return fmax(a, b); };
        largest = of_wave(largest, tx, larger64);
        if (tx > 64) {
            if ((threadIdx.x & 63) == 0) red64[threadIdx.x >> 6] = largest;
            __syncthreads();
            largest = of_waves(red64, tx, larger64);
        }
        const RowTo8<double> again8(largest);
        each([&](int c, double v) {
            const double one[1] = {v};
            int8_t q[1];
            again8(one, q);
            ((int8_t *)p.y)[row * p.ld_y + c] = q[0];
        });
        if (on && lane == 0) p.per_row[row] = scale(largest);
    }
}

// ------------------------------------------------------------------ gradient
struct Grad {
    const void *dy, *dsum, *sum, *weight;
    long ld_dy, ld_dsum, ld_sum;
    const float *inv_rms;
    void *dx;
    long ld_dx;
    float *dw;              // [workgroups][width] partial sums, or the gradient itself of one workgroup; NULL: not wanted
    long rows;
    int width, tx;
};

// Bound by memory: 8192 rows of 4096 bf16 with a gradient of the sum, 268 MB, in 51 - 54 us (5.0 - 5.3 TB/s) and 4 - 5 for the weight's partial sums.  A workgroup goes from row to row, the next one on its way,
// with its share of the weight's gradient in registers; 512 workgroups (256: 66 us, 1024: 52).
template <typename T, int HOLD, Way WAY>
__global__ __launch_bounds__(kMostLanes)
void norm_grad(Grad p)
{
    constexpr int n = Vec<T>::n;
    __shared__ float red[2][kMostLanes / 64];
    __shared__ float part[HOLD * kMostLanes * n];
    const int tx = p.tx, lane = (int)threadIdx.x & (tx - 1), ty = (int)blockDim.x >> __builtin_ctz(tx), line = (int)threadIdx.x >> __builtin_ctz(tx);
    const Row<T, WAY> at(p.width);
    const T *w = (const T *)p.weight;
    auto weights = [&](int i) {
        if (w) return at.load(w, i);
        Vec<T> one;
#pragma unroll
        for (int e = 0; e < n; ++e) one.v[e] = (T)1.f;
        return one;
    };
    Vec<T> by[HOLD];
    float dw[HOLD][n] = {};
#pragma unroll
    for (int u = 0; u < HOLD; ++u) {
        by[u] = {};
        if (lane + u * tx < at.count) by[u] = weights(lane + u * tx);
    }
    float *own = p.dw ? p.dw + (long)blockIdx.x * p.width : nullptr;
    const long step = (long)gridDim.x * ty;
    struct Pieces { Vec<T> g[HOLD], s[HOLD], add[HOLD]; float inv; } a, b;
    auto load = [&](Pieces &to, long row) {
        const bool on = row < p.rows;
        to.inv = on ? p.inv_rms[row] : 0.f;
#pragma unroll
        for (int u = 0; u < HOLD; ++u) {
            const int i = lane + u * tx;
            to.g[u] = to.s[u] = to.add[u] = {};
            if (on && i < at.count) {
                to.g[u] = at.load((const T *)p.dy + row * p.ld_dy, i);
                to.s[u] = at.load((const T *)p.sum + row * p.ld_sum, i);
                if (p.dsum) to.add[u] = at.load((const T *)p.dsum + row * p.ld_dsum, i);
            }
        }
    };
    // A row of this line, the next one on its way.  All lines of a workgroup go in step: their sums meet.
    auto step_of = [&](const Pieces &now, Pieces &next, long row, int turn) {
        const bool on = row < p.rows;
        load(next, row + step);
        float dot = 0.f;
#pragma unroll
        for (int u = 0; u < HOLD; ++u) {
            const int twice = at.twice(lane + u * tx);
#pragma unroll
            for (int e = 0; e < n; ++e)
                if (e >= twice) dot = fmaf((float)by[u].v[e] * (float)now.g[u].v[e], (float)now.s[u].v[e], dot);
        }
        const T *dy = (const T *)p.dy + row * p.ld_dy, *sum = (const T *)p.sum + row * p.ld_sum;
        if (WAY != kOverlap)
            for (int i = lane + HOLD * tx; on && i < at.count; i += tx) {
                const Vec<T> gi = at.load(dy, i), si = at.load(sum, i), wi = weights(i);
#pragma unroll
                for (int e = 0; e < n; ++e) dot = fmaf((float)wi.v[e] * (float)gi.v[e], (float)si.v[e], dot);
            }
        const auto plus = [](float a, float b) { return a + b; };
        dot = of_wave(dot, tx, plus);
        if (tx > 64) {
            if ((threadIdx.x & 63) == 0) red[turn][threadIdx.x >> 6] = dot;
            __syncthreads();
            dot = of_waves(red[turn], tx, plus);
        }
        if (!on) return;
        const float inv = now.inv, back = inv * (inv * (dot / (float)p.width));         // inv^2 alone may be beyond fp32, or too small for its 24 bits
        auto write = [&](int i, const Vec<T> &gi, const Vec<T> &si, const Vec<T> &wi, const Vec<T> &ai) {
            Vec<T> out;
#pragma unroll
            for (int e = 0; e < n; ++e) {
                const float v = inv * ((float)wi.v[e] * (float)gi.v[e] - (float)si.v[e] * back);
                out.v[e] = narrow<T>(p.dsum ? v + (float)ai.v[e] : v);
            }
            at.store((T *)p.dx + row * p.ld_dx, i, out.v);
        };
#pragma unroll
        for (int u = 0; u < HOLD; ++u) {
            if (lane + u * tx < at.count) write(lane + u * tx, now.g[u], now.s[u], by[u], now.add[u]);
#pragma unroll
            for (int e = 0; e < n; ++e) dw[u][e] = fmaf((float)now.g[u].v[e], (float)now.s[u].v[e] * inv, dw[u][e]);
        }
        // pieces that no lane holds: a row has the whole workgroup then, and their partial sums stay in memory, each a lane's own
        if (WAY != kOverlap)
            for (int i = lane + HOLD * tx; i < at.count; i += tx) {
                const Vec<T> gi = at.load(dy, i), si = at.load(sum, i), wi = weights(i);
                Vec<T> ai = {};
                if (p.dsum) ai = at.load((const T *)p.dsum + row * p.ld_dsum, i);
                if (own)
#pragma unroll
                    for (int e = 0; e < n; ++e)
                        if (i * n + e < p.width) own[i * n + e] = fmaf((float)gi.v[e], (float)si.v[e] * inv, row == (long)blockIdx.x ? 0.f : own[i * n + e]);
                write(i, gi, si, wi, ai);
            }
    };
    long row = (long)blockIdx.x * ty + line;
    load(a, row);
    for (long row0 = (long)blockIdx.x * ty; row0 < p.rows; row0 += 2 * step, row += 2 * step) {
        step_of(a, b, row, 0);
        if (row0 + step < p.rows) step_of(b, a, row + step, 1);
    }
    if (!own) return;
    // the lines' sums: those of a wave in its registers, the waves' one after the other (195 rows of 64 in bf16: 13 us with all 32 lines one after the other, 5 like this)
    for (int o = tx; o < 64; o *= 2)
#pragma unroll
        for (int u = 0; u < HOLD; ++u)
#pragma unroll
            for (int e = 0; e < n; ++e) dw[u][e] += __shfl_xor(dw[u][e], o);
    const int sums = tx < 64 ? (int)blockDim.x >> 6 : ty, mine = tx < 64 ? (int)threadIdx.x >> 6 : line;
    const bool first = tx >= 64 || ((int)threadIdx.x & 63) < tx;
    for (int l = 0; l < sums; ++l) {
        if (mine == l && first)
#pragma unroll
            for (int u = 0; u < HOLD; ++u)
#pragma unroll
                for (int e = 0; e < n; ++e) {
                    float &to = part[(e * HOLD + u) * tx + lane];
                    to = l == 0 ? dw[u][e] : to + dw[u][e];
                }
        __syncthreads();
    }
    const int held = min(p.width, HOLD * tx * n);
    for (int c = threadIdx.x; c < held; c += blockDim.x) {
        const int i = c / n, u = i / tx;
        own[c] = part[((c - at.first(i)) * HOLD + u) * tx + i - u * tx];
    }
    if (p.rows == 0)
        for (int c = held + threadIdx.x; c < p.width; c += blockDim.x) own[c] = 0.f;
}

// dw[c] = the sum of part[0 .. parts][c]: kCols columns a workgroup, a part of the lines each thread, joined in the LDS.
constexpr int kCols = 16, kLines = 64;
__global__ __launch_bounds__(kCols * kLines)
void norm_grad_weight(const float *__restrict__ part, int parts, int width, float *__restrict__ dw)
{
    __shared__ float red[kLines][kCols + 1];
    const int col = (int)threadIdx.x % kCols, line = (int)threadIdx.x / kCols;
    const long c = (long)blockIdx.x * kCols + col;
    float sum = 0.f;
    if (c < width)
#pragma unroll 8
        for (int i = line; i < parts; i += kLines) sum += part[(long)i * width + c];
    red[line][col] = sum;
    __syncthreads();
    for (int half = kLines / 2; half > 0; half /= 2) {
        if (line < half) red[line][col] += red[line + half][col];
        __syncthreads();
    }
    if (line == 0 && c < width) dw[c] = red[0][col];
}

// ------------------------------------------------------------------ host side
using opevo::launch;

// `tx` lanes to a row of `pieces`, at most `lanes` of them, `hold` pieces a lane.
struct Shape { int tx, hold; };
Shape shape_of(int64_t pieces, int lanes, int most)
{
    int tx = 1, hold = 1;
    while (tx < lanes && tx < pieces) tx *= 2;
    while (hold < most && (int64_t)tx * hold < pieces) hold *= 2;
    return {tx, hold};
}

int check_norm(const char *who, const Norm &p, int dtype, int64_t rows, int64_t width)
{
    if (!known(dtype)) return fail(OPEVO_E_ARG, "%s: unknown element type %d", who, dtype);
    if (rows < 0 || rows > INT32_MAX) return fail(OPEVO_E_ARG, "%s: %lld rows", who, (long long)rows);
    if (!(p.eps >= 0.f) || p.eps > FLT_MAX) return fail(OPEVO_E_ARG, "%s: eps is negative, infinite or not a number", who);
    if (rows == 0) return OPEVO_OK;
    const size_t size = size_of(dtype);
    if (int rc = check_rows(who, "x", p.x, p.ld_x, width, size)) return rc;
    if (p.residual)
        if (int rc = check_rows(who, "residual", p.residual, p.ld_residual, width, size)) return rc;
    if (p.residual && !p.sum) return fail(OPEVO_E_ARG, "%s: sum is NULL, but there is a residual", who);
    if (p.sum)
        if (int rc = check_rows(who, "sum", p.sum, p.ld_sum, width, size)) return rc;
    if (!aligned(p.weight, size)) return fail(OPEVO_E_ARG, "%s: weight is not aligned to its elements", who);
    return OPEVO_OK;
}

template <typename T, bool TO8>
int run_norm(Norm p, hipStream_t stream)
{
    constexpr int n = Vec<T>::n;
    const int64_t pieces = (p.width + n - 1) / n;
    const Shape l = shape_of(pieces, kMostLanes, 4);
    const bool held = pieces <= (int64_t)l.tx * l.hold;
    p.tx = l.tx;
    const int threads = std::max(l.tx, kThreads), ty = threads / l.tx;
    auto *k = p.width % n == 0 ? (l.hold == 1 ? norm_rows<T, 1, TO8, kWhole> : l.hold == 2 ? norm_rows<T, 2, TO8, kWhole> : norm_rows<T, 4, TO8, kWhole>)
              : p.width > n && held ? (l.hold == 1 ? norm_rows<T, 1, TO8, kOverlap> : l.hold == 2 ? norm_rows<T, 2, TO8, kOverlap> : norm_rows<T, 4, TO8, kOverlap>)
                                    : norm_rows<T, 1, TO8, kRest>;
    return launch("norm_rows launch", k, spread((p.rows + ty - 1) / ty, 1, threads), dim3(threads), stream, p);
}
template <typename T> int run_plain(const Norm &p, hipStream_t stream) { return run_norm<T, false>(p, stream); }
template <typename T> int run_to8(const Norm &p, hipStream_t stream) { return run_norm<T, true>(p, stream); }

// Workgroups of the gradient: each goes through its rows with the weight's gradient in registers.  Half as many of 512 lanes: they leave half as many partial sums (norm and gradient, 501 rows of 5288
// bf16 26.0 -> 20.6 us, 1000 of 8192 37.9 -> 31.7, 8192 of 8192 201 -> 196; for shorter rows they take longer, 1001 of 1000 fp32 14.8 -> 16.3).
constexpr int64_t kGroups = 512;
int64_t groups_of(int64_t rows, int ty, int64_t most) { return std::max<int64_t>(1, std::min<int64_t>(most, (rows + ty - 1) / ty)); }

template <typename T>
int run_grad(Grad p, float *dweight, float *workspace, hipStream_t stream)
{
    constexpr int n = Vec<T>::n;
    const int64_t pieces = (p.width + n - 1) / n;
    // two pieces on 256 lanes rather than one on 512 (8192 rows of 4096 bf16: 47 us and 65), which are for longer rows
    const Shape l = shape_of(pieces, pieces > 2 * kThreads ? kMostLanes : kThreads, 2);
    const bool held = pieces <= (int64_t)l.tx * l.hold;
    p.tx = l.tx;
    const int threads = std::max(l.tx, kThreads);
    const int64_t groups = groups_of(p.rows, threads / l.tx, l.tx > kThreads ? kGroups / 2 : kGroups);
    p.dw = !dweight ? nullptr : groups == 1 ? dweight : workspace;
    auto *k = p.width % n == 0 ? (l.hold == 1 ? norm_grad<T, 1, kWhole> : norm_grad<T, 2, kWhole>)
              : p.width > n && held ? (l.hold == 1 ? norm_grad<T, 1, kOverlap> : norm_grad<T, 2, kOverlap>) : norm_grad<T, 1, kRest>;
    if (int rc = launch("norm_grad launch", k, dim3((unsigned)groups), dim3(threads), stream, p)) return rc;
    if (!dweight || groups == 1) return OPEVO_OK;
    return launch("norm_grad_weight launch", norm_grad_weight, dim3((p.width + kCols - 1) / kCols), dim3(kCols * kLines), stream, workspace, (int)groups, p.width, dweight);
}

}  // namespace

extern "C" int opevo_norm_rows(const void *x, int64_t ld_x, const void *residual, int64_t ld_residual, const void *weight, float eps, int dtype, int64_t rows,
                               int64_t width, void *sum, int64_t ld_sum, void *y, int64_t ld_y, float *inv_rms, void *stream)
{
    const char *who = "norm_rows";
    Norm p = {x, residual, weight, (long)ld_x, (long)ld_residual, sum, (long)ld_sum, y, (long)ld_y, inv_rms, (long)rows, (int)width, 0, eps};
    if (int rc = check_norm(who, p, dtype, rows, width)) return rc;
    if (rows == 0) return OPEVO_OK;
    if (int rc = check_rows(who, "y", y, ld_y, width, size_of(dtype))) return rc;
    if (!aligned(inv_rms, 4)) return fail(OPEVO_E_ARG, "%s: inv_rms is not aligned to 4 bytes", who);
    return BY_DTYPE(dtype, run_plain, p, static_cast<hipStream_t>(stream));
}

extern "C" int opevo_norm_rows_i8(const void *x, int64_t ld_x, const void *residual, int64_t ld_residual, const void *weight, float eps, int dtype, int64_t rows,
                                  int64_t width, void *sum, int64_t ld_sum, int8_t *q, int64_t ld_q, float *scale, void *stream)
{
    const char *who = "norm_rows_i8";
    Norm p = {x, residual, weight, (long)ld_x, (long)ld_residual, sum, (long)ld_sum, q, (long)ld_q, scale, (long)rows, (int)width, 0, eps};
    if (int rc = check_norm(who, p, dtype, rows, width)) return rc;
    if (rows == 0) return OPEVO_OK;
    if (int rc = check_rows(who, "q", q, ld_q, width, 1)) return rc;
    if (int rc = check_words(who, "scale", scale)) return rc;
    return BY_DTYPE(dtype, run_to8, p, static_cast<hipStream_t>(stream));
}

static int check_size(const char *who, int64_t rows, int64_t width)
{
    if (rows < 0 || rows > INT32_MAX) return fail(OPEVO_E_ARG, "%s: %lld rows", who, (long long)rows);
    if (width < 1 || width > (1 << 24)) return fail(OPEVO_E_ARG, "%s: rows of %lld elements (1 to 2^24)", who, (long long)width);
    return OPEVO_OK;
}

extern "C" int opevo_norm_rows_grad_workspace(int64_t rows, int64_t width, size_t *bytes)
{
    if (!bytes) return fail(OPEVO_E_ARG, "norm_rows_grad_workspace: bytes is NULL");
    if (int rc = check_size("norm_rows_grad_workspace", rows, width)) return rc;
    const int64_t groups = std::min(kGroups, rows);
    *bytes = groups <= 1 ? 0 : sizeof(float) * (size_t)(groups * width);
    return OPEVO_OK;
}

extern "C" int opevo_norm_rows_grad(const void *dy, int64_t ld_dy, const void *dsum, int64_t ld_dsum, const void *sum, int64_t ld_sum, const void *weight,
                                    const float *inv_rms, int dtype, int64_t rows, int64_t width, void *dx, int64_t ld_dx, float *dweight, void *workspace,
                                    size_t workspace_bytes, void *stream)
{
    const char *who = "norm_rows_grad";
    if (!known(dtype)) return fail(OPEVO_E_ARG, "%s: unknown element type %d", who, dtype);
    if (int rc = check_size(who, rows, width)) return rc;
    const size_t size = size_of(dtype);
    if (dweight && !aligned(dweight, 4)) return fail(OPEVO_E_ARG, "%s: dweight is not aligned to 4 bytes", who);
    if (rows > 0) {
        if (int rc = check_rows(who, "dy", dy, ld_dy, width, size)) return rc;
        if (dsum)
            if (int rc = check_rows(who, "dsum", dsum, ld_dsum, width, size)) return rc;
        if (int rc = check_rows(who, "sum", sum, ld_sum, width, size)) return rc;
        if (int rc = check_rows(who, "dx", dx, ld_dx, width, size)) return rc;
        if (int rc = check_words(who, "inv_rms", inv_rms)) return rc;
        if (!aligned(weight, size)) return fail(OPEVO_E_ARG, "%s: weight is not aligned to its elements", who);
    }
    size_t need = 0;
    if (int rc = opevo_norm_rows_grad_workspace(rows, width, &need)) return rc;
    if (dweight && need && (!workspace || !aligned(workspace, 4) || workspace_bytes < need))
        return fail(OPEVO_E_ARG, "%s: the workspace holds %zu bytes of the %zu it takes, or is not aligned to 4 bytes", who, workspace ? workspace_bytes : 0, need);
    if (rows == 0 && !dweight) return OPEVO_OK;
    Grad p = {dy, dsum, sum, weight, (long)ld_dy, (long)ld_dsum, (long)ld_sum, inv_rms, dx, (long)ld_dx, nullptr, (long)rows, (int)width, 0};
    return BY_DTYPE(dtype, run_grad, p, dweight, static_cast<float *>(workspace), static_cast<hipStream_t>(stream));
}
