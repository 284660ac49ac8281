// Routing of an expert layer: tokens to the rows of their experts (dispatch), rows back to their tokens with weights
// (combine), the gradients of both, and rows of numbers to 8-bit integers with a scale each.
//
// T tokens have k slots each; slot s = t * k + j names an expert or none that is held here.  The stable sort of the slots by
// expert gives every held slot a row; everything else is rows copied or summed.  None of it has arithmetic to speak of: the
// floor is the bytes, and for a few tokens the launch.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdint>

#include "kernel.hpp"
#include "narrow.hpp"

namespace {

constexpr int kThreads = 256;
constexpr int kMaxExperts = OPEVO_ROUTE_MAX_EXPERTS;

template <typename T> struct Bits;
template <> struct Bits<float> { typedef uint32_t type; };
template <> struct Bits<_Float16> { typedef uint16_t type; };
template <> struct Bits<__bf16> { typedef uint16_t type; };

// 16 bytes of a row.  Rows start wherever the caller's row length puts them, so all such accesses are made for any alignment (the hardware's
// 16-byte loads and stores take any address; the compiler is told nothing more).
template <typename T> struct Vec {
    static constexpr int n = 16 / sizeof(T);
    T v[n];
};
template <typename T> __device__ __forceinline__ Vec<T> load16(const T *p)
{
    Vec<T> r;
    __builtin_memcpy(&r, p, 16);
    return r;
}
template <typename T> __device__ __forceinline__ void store16(T *p, const Vec<T> &r) { __builtin_memcpy(p, &r, 16); }

// ------------------------------------------------------------------ the sort
// How many slots of a chunk go to each expert: counts[chunk][expert].
__global__ __launch_bounds__(kThreads)
void route_count(const int *__restrict__ expert, long slots, int chunk, int experts, int *__restrict__ counts)
{
    __shared__ int hist[kMaxExperts];
    for (int e = threadIdx.x; e < experts; e += kThreads) hist[e] = 0;
    __syncthreads();
    const long first = (long)blockIdx.x * chunk, last = first + chunk < slots ? first + chunk : slots;
    for (long s = first + threadIdx.x; s < last; s += kThreads) {
        const unsigned e = expert[s];
        if (e < (unsigned)experts) atomicAdd(&hist[e], 1);
    }
    __syncthreads();
    for (int e = threadIdx.x; e < experts; e += kThreads) counts[(long)blockIdx.x * experts + e] = hist[e];
}

struct Route {
    const int *expert;
    long tokens;
    int k, experts;
    const int *counts;      // NULL: every workgroup counts all slots itself
    int chunk, chunks;
    int tokens_per_block;
    int *offsets, *row_of_slot;
};

// Rows of this workgroup's slots into place[] (-1: none), from the slots' experts alone: a slot's row is the number of slots of
// lower experts, plus the earlier slots of its own.  Earlier slots are those of earlier chunks (counted by route_count, a column sum), those of
// its chunk before this workgroup's first (counted here), and those of this workgroup before it.  Integer counts: any order gives the same.
// Returns the number of slots that have a row.
__device__ __forceinline__ int route_rows(const Route &r, long first_slot, int own, int *place, int *mine, int *total, int *before, bool writes)
{
    const int tid = threadIdx.x;
    const long slots = r.tokens * r.k;
    for (int e = tid; e < r.experts; e += kThreads) total[e] = before[e] = 0;
    if (tid < own) mine[tid] = r.expert[first_slot + tid];
    __syncthreads();
    if (r.counts) {
        const int at = (int)(first_slot / r.chunk);
        for (int i = tid; i < r.chunks * r.experts; i += kThreads) {
            const int n = r.counts[i], c = i / r.experts, e = i - c * r.experts;
            if (n) {
                atomicAdd(&total[e], n);
                if (c < at) atomicAdd(&before[e], n);
            }
        }
        for (long s = (long)at * r.chunk + tid; s < first_slot; s += kThreads) {
            const unsigned e = r.expert[s];
            if (e < (unsigned)r.experts) atomicAdd(&before[e], 1);
        }
    } else {
        for (long s = tid; s < slots; s += kThreads) {
            const unsigned e = r.expert[s];
            if (e < (unsigned)r.experts) {
                atomicAdd(&total[e], 1);
                if (s < first_slot) atomicAdd(&before[e], 1);
            }
        }
    }
    __syncthreads();
    __shared__ int held;
    if (tid < 64) {                         // exclusive sums over the experts, 64 at a time
        int run = 0;
        for (int e0 = 0; e0 < r.experts; e0 += 64) {
            const int e = e0 + tid, n = e < r.experts ? total[e] : 0;
            int sum = n;
#pragma unroll
            for (int o = 1; o < 64; o <<= 1) {
                const int up = __shfl_up(sum, o);
                if (tid >= o) sum += up;
            }
            if (e < r.experts) {
                before[e] += run + sum - n;
                if (writes) r.offsets[e] = run + sum - n;
            }
            run += __shfl(sum, 63);
        }
        if (tid == 0) {
            held = run;
            if (writes) r.offsets[r.experts] = run;
        }
    }
    __syncthreads();
    if (tid < own) {
        const int e = mine[tid];
        int row = -1;
        if ((unsigned)e < (unsigned)r.experts) {
            row = before[e];
            for (int i = 0; i < tid; ++i) row += mine[i] == e;
        }
        place[tid] = row;
    }
    __syncthreads();
    return held;
}

// Threads of a workgroup over rows of `vecs` pieces: `tx` lanes (a power of two) side by side on a row, the others on further rows.
struct Lay { int tx, ty; };
static Lay lay_out(int64_t vecs)
{
    int tx = 1;
    while (tx < kThreads && tx < vecs) tx *= 2;
    return {tx, kThreads / tx};
}

// ------------------------------------------------------------------ dispatch
template <typename T>
__global__ __launch_bounds__(kThreads)
void route_dispatch(Route r, const T *__restrict__ x, long ld_x, int width, int tx, T *__restrict__ rows, long ld_rows)
{
    __shared__ int place[kThreads], mine[kThreads], total[kMaxExperts], before[kMaxExperts];
    const long first = (long)blockIdx.x * r.tokens_per_block;
    const int tokens = (int)(r.tokens - first < r.tokens_per_block ? r.tokens - first : r.tokens_per_block), own = tokens * r.k;
    const int held = route_rows(r, first * r.k, own, place, mine, total, before, blockIdx.x == 0 && blockIdx.y == 0);
    if (blockIdx.y == 0 && (int)threadIdx.x < own) r.row_of_slot[first * r.k + threadIdx.x] = place[threadIdx.x];
    const int lane = threadIdx.x % tx, ty = kThreads / tx, line = threadIdx.x / tx;
    const int vecs = width / Vec<T>::n, step = tx * gridDim.y, start = blockIdx.y * tx + lane;
    const int tail0 = vecs * Vec<T>::n;
    for (int t = line; t < tokens; t += ty) {
        const T *src = x + (first + t) * ld_x;
        for (int c = start; c < vecs; c += step) {
            const Vec<T> v = load16(src + c * Vec<T>::n);
            for (int j = 0; j < r.k; ++j) {
                const int row = place[t * r.k + j];
                if (row >= 0) store16(rows + row * ld_rows + c * Vec<T>::n, v);
            }
        }
        for (int c = tail0 + start; c < width; c += step) {
            const T v = src[c];
            for (int j = 0; j < r.k; ++j) {
                const int row = place[t * r.k + j];
                if (row >= 0) rows[row * ld_rows + c] = v;
            }
        }
    }
    // rows that no slot goes to
    const Vec<T> zero = {};
    for (long row = held + (long)blockIdx.x * ty + line; row < r.tokens * r.k; row += (long)gridDim.x * ty) {
        for (int c = start; c < vecs; c += step) store16(rows + row * ld_rows + c * Vec<T>::n, zero);
        for (int c = tail0 + start; c < width; c += step) rows[row * ld_rows + c] = (T)0.f;
    }
}

// ------------------------------------------------------------------ rows to 8 bits
// The largest magnitude as its bits: for numbers without a sign the order of the bits is that of the values, and infinities and
// NaNs come last.
constexpr unsigned kInfinite = 0x7f800000u;

template <typename T> __device__ __forceinline__ unsigned magnitude(const Vec<T> &v)
{
    unsigned m = 0;
#pragma unroll
    for (int i = 0; i < Vec<T>::n; ++i) m = max(m, __float_as_uint((float)v.v[i]) & 0x7fffffffu);
    return m;
}

// q = round(127 x / a), a the row's largest magnitude.  With 127 x computed first (exact for 16-bit inputs: 11 + 7 bits) and one
// division, the quotient of two numbers of at most 18 and 11 bits is a tie in fp32 only where it is one exactly, so the result is the
// rounding of the exact quotient; fp32 inputs may differ from it where the quotient is within 2^-24 of a tie.
struct Quantizer { float a, pre; bool finite; };
__device__ __forceinline__ Quantizer quantizer(unsigned m)
{
    const float a = __uint_as_float(m);
    const float pre = a > 1e30f ? 0.0078125f : 1.f;        // 127 x stays finite
    return {a * pre, pre, m < kInfinite};
}
__device__ __forceinline__ int quantize(float x, const Quantizer &z)
{
    return z.finite && z.a > 0.f ? (int)rintf(127.f * (x * z.pre) / z.a) : 0;
}
__device__ __forceinline__ float scale_of(unsigned m)
{
    return m < kInfinite ? __uint_as_float(m) / 127.f : __uint_as_float(0x7fc00000u);
}
template <typename T> __device__ __forceinline__ void quantize16(const Vec<T> &v, const Quantizer &z, int8_t (&q)[Vec<T>::n])
{
#pragma unroll
    for (int i = 0; i < Vec<T>::n; ++i) q[i] = (int8_t)quantize((float)v.v[i], z);
}

// The maximum over the tx lanes of a row (red: one word a wave).
__device__ __forceinline__ unsigned row_max(unsigned m, int tx, unsigned *red)
{
    for (int o = 1; o < tx && o < 64; o <<= 1) m = max(m, (unsigned)__shfl_xor((int)m, o));
    if (tx > 64) {
        __syncthreads();
        if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = m;
        __syncthreads();
        const int w0 = threadIdx.x / tx * (tx / 64);
        for (int w = 0; w < tx / 64; ++w) m = max(m, red[w0 + w]);
    }
    return m;
}

template <typename T>
__device__ __forceinline__ unsigned scan_row(const T *src, int width, int lane, int tx)
{
    const int vecs = width / Vec<T>::n;
    unsigned m = 0;
    for (int c = lane; c < vecs; c += tx) m = max(m, magnitude(load16(src + c * Vec<T>::n)));
    for (int c = vecs * Vec<T>::n + lane; c < width; c += tx) m = max(m, __float_as_uint((float)src[c]) & 0x7fffffffu);
    return m;
}

template <typename T>
__global__ __launch_bounds__(kThreads)
void quantize_rows(const T *__restrict__ x, long ld_x, long rows, int width, int tx, int8_t *__restrict__ q, long ld_q, float *__restrict__ scale)
{
    __shared__ unsigned red[kThreads / 64];
    const int lane = threadIdx.x % tx, ty = kThreads / tx, vecs = width / Vec<T>::n;
    const long row = (long)blockIdx.x * ty + threadIdx.x / tx;
    const bool on = row < rows;
    const T *src = x + (on ? row : 0) * ld_x;
    const unsigned m = row_max(on ? scan_row(src, width, lane, tx) : 0u, tx, red);
    if (!on) return;
    const Quantizer z = quantizer(m);
    int8_t *dst = q + row * ld_q;
    for (int c = lane; c < vecs; c += tx) {
        int8_t out[Vec<T>::n];
        quantize16(load16(src + c * Vec<T>::n), z, out);
        __builtin_memcpy(dst + c * Vec<T>::n, out, sizeof out);
    }
    for (int c = vecs * Vec<T>::n + lane; c < width; c += tx) dst[c] = (int8_t)quantize((float)src[c], z);
    if (lane == 0) scale[row] = scale_of(m);
}

template <typename T>
__global__ __launch_bounds__(kThreads)
void route_dispatch_i8(Route r, const T *__restrict__ x, long ld_x, int width, int tx, int8_t *__restrict__ q, long ld_q, float *__restrict__ scale)
{
    __shared__ int place[kThreads], mine[kThreads], total[kMaxExperts], before[kMaxExperts];
    __shared__ unsigned red[kThreads / 64];
    const long first = (long)blockIdx.x * r.tokens_per_block;
    const int tokens = (int)(r.tokens - first < r.tokens_per_block ? r.tokens - first : r.tokens_per_block), own = tokens * r.k;
    const int held = route_rows(r, first * r.k, own, place, mine, total, before, blockIdx.x == 0);
    if ((int)threadIdx.x < own) r.row_of_slot[first * r.k + threadIdx.x] = place[threadIdx.x];
    const int lane = threadIdx.x % tx, ty = kThreads / tx, line = threadIdx.x / tx;
    const int vecs = width / Vec<T>::n;
    for (int t0 = 0; t0 < tokens; t0 += ty) {
        const int t = t0 + line;
        const bool on = t < tokens;
        const T *src = x + (first + (on ? t : 0)) * ld_x;
        const unsigned m = row_max(on ? scan_row(src, width, lane, tx) : 0u, tx, red);
        if (!on) continue;                  // every lane of a row's line alike; a line longer than a wave is the whole workgroup's trip
        const Quantizer z = quantizer(m);
        for (int c = lane; c < vecs; c += tx) {
            int8_t out[Vec<T>::n];
            quantize16(load16(src + c * Vec<T>::n), z, out);
            for (int j = 0; j < r.k; ++j) {
                const int row = place[t * r.k + j];
                if (row >= 0) __builtin_memcpy(q + row * ld_q + c * Vec<T>::n, out, sizeof out);
            }
        }
        for (int c = vecs * Vec<T>::n + lane; c < width; c += tx) {
            const int8_t out = (int8_t)quantize((float)src[c], z);
            for (int j = 0; j < r.k; ++j) {
                const int row = place[t * r.k + j];
                if (row >= 0) q[row * ld_q + c] = out;
            }
        }
        for (int j = lane; j < r.k; j += tx) {
            const int row = place[t * r.k + j];
            if (row >= 0) scale[row] = scale_of(m);
        }
    }
    for (long row = held + (long)blockIdx.x * ty + line; row < r.tokens * r.k; row += (long)gridDim.x * ty) {
        for (int c = lane; c < width; c += tx) q[row * ld_q + c] = 0;
        if (lane == 0) scale[row] = 0.f;
    }
}

// ------------------------------------------------------------------ combine
// y[t] = sum_j w[t, j] rows[row_of_slot[t, j]], j ascending, in fp32, rounded once; a slot without a row adds nothing, whatever its weight.
template <typename T>
__global__ __launch_bounds__(kThreads)
void route_combine(const T *__restrict__ rows, long ld_rows, const float *__restrict__ weight, const int *__restrict__ row_of_slot,
                   long tokens, int k, int width, int tx, T *__restrict__ y, long ld_y)
{
    const int lane = threadIdx.x % tx, ty = kThreads / tx;
    const long t = (long)blockIdx.x * ty + threadIdx.x / tx, slots = tokens * k;
    if (t >= tokens) return;
    const int vecs = width / Vec<T>::n, step = tx * gridDim.y, start = blockIdx.y * tx + lane;
    for (int c = start; c < vecs; c += step) {
        float sum[Vec<T>::n] = {};
        for (int j = 0; j < k; ++j) {
            const int row = row_of_slot[t * k + j];
            if ((unsigned)row >= (unsigned long)slots) continue;
            const float w = weight ? weight[t * k + j] : 1.f;
            const Vec<T> v = load16(rows + row * ld_rows + c * Vec<T>::n);
#pragma unroll
            for (int i = 0; i < Vec<T>::n; ++i) sum[i] = fmaf(w, (float)v.v[i], sum[i]);
        }
        Vec<T> out;
#pragma unroll
        for (int i = 0; i < Vec<T>::n; ++i) out.v[i] = narrow<T>(sum[i]);
        store16(y + t * ld_y + c * Vec<T>::n, out);
    }
    for (int c = vecs * Vec<T>::n + start; c < width; c += step) {
        float sum = 0.f;
        for (int j = 0; j < k; ++j) {
            const int row = row_of_slot[t * k + j];
            if ((unsigned)row >= (unsigned long)slots) continue;
            sum = fmaf(weight ? weight[t * k + j] : 1.f, (float)rows[row * ld_rows + c], sum);
        }
        y[t * ld_y + c] = narrow<T>(sum);
    }
}

// drows[row_of_slot[s]] = w[s] dy[s / k], dw[s] = <dy[s / k], rows[row_of_slot[s]]>; rows from offsets[experts] on get zeros, slots without a row dw = 0.
template <typename T>
__global__ __launch_bounds__(kThreads)
void route_combine_grad(const T *__restrict__ dy, long ld_dy, const T *__restrict__ rows, long ld_rows, const float *__restrict__ weight,
                        const int *__restrict__ row_of_slot, const int *__restrict__ held_at, long tokens, int k, int width, int tx,
                        T *__restrict__ drows, long ld_drows, float *__restrict__ dweight)
{
    __shared__ float red[kThreads / 64];
    const int lane = threadIdx.x % tx, ty = kThreads / tx, line = threadIdx.x / tx;
    const long t = (long)blockIdx.x * ty + line, slots = tokens * k;
    const bool on = t < tokens;
    const int vecs = width / Vec<T>::n;
    for (int j = 0; j < k; ++j) {
        const int row = on ? row_of_slot[t * k + j] : -1;
        const bool has = (unsigned)row < (unsigned long)slots;
        const float w = has ? weight[t * k + j] : 0.f;
        float dot = 0.f;
        if (has) {
            for (int c = lane; c < vecs; c += tx) {
                const Vec<T> g = load16(dy + t * ld_dy + c * Vec<T>::n), v = load16(rows + row * ld_rows + c * Vec<T>::n);
                Vec<T> out;
#pragma unroll
                for (int i = 0; i < Vec<T>::n; ++i) {
                    dot = fmaf((float)g.v[i], (float)v.v[i], dot);
                    out.v[i] = narrow<T>(w * (float)g.v[i]);
                }
                store16(drows + row * ld_drows + c * Vec<T>::n, out);
            }
            for (int c = vecs * Vec<T>::n + lane; c < width; c += tx) {
                const float g = (float)dy[t * ld_dy + c];
                dot = fmaf(g, (float)rows[row * ld_rows + c], dot);
                drows[row * ld_drows + c] = narrow<T>(w * g);
            }
        }
        for (int o = 1; o < tx && o < 64; o <<= 1) dot += __shfl_xor(dot, o);
        if (tx > 64) {
            __syncthreads();
            if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = dot;
            __syncthreads();
            const int w0 = line * (tx / 64);
            dot = 0.f;
            for (int i = 0; i < tx / 64; ++i) dot += red[w0 + i];
        }
        if (on && lane == 0) dweight[t * k + j] = dot;
    }
    const Vec<T> zero = {};
    const int held = *held_at;
    for (long row = (held > 0 ? held : 0) + (long)blockIdx.x * ty + line; row < slots; row += (long)gridDim.x * ty) {
        for (int c = lane; c < vecs; c += tx) store16(drows + row * ld_drows + c * Vec<T>::n, zero);
        for (int c = vecs * Vec<T>::n + lane; c < width; c += tx) drows[row * ld_drows + c] = (T)0.f;
    }
}

// ------------------------------------------------------------------ host side
using opevo::fail;

bool aligned(const void *p, size_t to) { return reinterpret_cast<uintptr_t>(p) % to == 0; }
size_t size_of(int dtype) { return dtype == OPEVO_F32 ? 4 : 2; }
bool known(int dtype) { return dtype == OPEVO_F32 || dtype == OPEVO_BF16 || dtype == OPEVO_F16; }

int launched(const char *what)
{
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? OPEVO_OK : opevo::hip_fail(e, what);
}

int check_route(const char *who, int64_t tokens, int k, int experts)
{
    if (tokens < 0 || k < 1 || k > OPEVO_ROUTE_MAX_SLOTS || tokens > INT32_MAX / k)
        return fail(OPEVO_E_ARG, "%s: tokens %lld with %d slots each (1 to %d, fewer than 2^31 in all)", who, (long long)tokens, k, OPEVO_ROUTE_MAX_SLOTS);
    if (experts < 1 || experts > kMaxExperts) return fail(OPEVO_E_ARG, "%s: %d experts (1 to %d)", who, experts, kMaxExperts);
    return OPEVO_OK;
}
// rows of `width` elements, `ld` apart
int check_rows(const char *who, const char *name, const void *p, int64_t ld, int64_t width, size_t bytes)
{
    if (!p) return fail(OPEVO_E_ARG, "%s: %s is NULL", who, name);
    if (!aligned(p, bytes)) return fail(OPEVO_E_ARG, "%s: %s is not aligned to its elements", who, name);
    if (width < 1 || width > (1 << 24)) return fail(OPEVO_E_ARG, "%s: rows of %lld elements (1 to 2^24)", who, (long long)width);
    if (ld < width || ld > ((int64_t)1 << 40)) return fail(OPEVO_E_ARG, "%s: rows of %s are %lld apart, shorter than their %lld elements or beyond 2^40", who, name, (long long)ld, (long long)width);
    return OPEVO_OK;
}
int check_words(const char *who, const char *name, const void *p)
{
    return p && aligned(p, 4) ? OPEVO_OK : fail(OPEVO_E_ARG, "%s: %s is NULL or not aligned to 4 bytes", who, name);
}

// Up to this many slots every workgroup counts them all itself; beyond, route_count does it chunk by chunk.
constexpr int64_t kCountAlone = 4096;
// A workgroup reads chunks * experts counts and half a chunk of slots on average.
int64_t chunk_of(int64_t slots, int experts)
{
    int64_t chunk = 256;
    while (chunk < 8192 && chunk * chunk < 2 * slots * experts) chunk *= 2;
    return chunk;
}

// Fills r and, where it takes one, launches the count.
int plan_route(const char *who, const int32_t *expert, int64_t tokens, int k, int experts, int32_t *offsets, int32_t *row_of_slot,
               void *workspace, size_t workspace_bytes, hipStream_t stream, Route *r)
{
    const int64_t slots = tokens * k;
    r->expert = expert; r->tokens = tokens; r->k = k; r->experts = experts;
    r->counts = nullptr; r->chunk = 1; r->chunks = 0;
    r->offsets = offsets; r->row_of_slot = row_of_slot;
    if (slots > kCountAlone) {
        r->chunk = (int)chunk_of(slots, experts);
        r->chunks = (int)((slots + r->chunk - 1) / r->chunk);
        const size_t need = sizeof(int) * (size_t)r->chunks * experts;
        if (!workspace || !aligned(workspace, 4) || workspace_bytes < need)
            return fail(OPEVO_E_ARG, "%s: the workspace holds %zu bytes of the %zu it takes, or is not aligned to 4 bytes", who, workspace ? workspace_bytes : 0, need);
        hipLaunchKernelGGL(route_count, dim3(r->chunks), dim3(kThreads), 0, stream, expert, (long)slots, r->chunk, experts, static_cast<int *>(workspace));
        if (int rc = launched("route_count launch")) return rc;
        r->counts = static_cast<const int *>(workspace);
    }
    // as many tokens a workgroup as leave 1024 workgroups, and as have a slot for each thread
    r->tokens_per_block = (int)std::max<int64_t>(1, std::min<int64_t>(kThreads / k, tokens / 1024));
    return OPEVO_OK;
}

template <typename T>
int run_dispatch(const Route &r, const void *x, int64_t ld_x, int64_t width, void *rows, int64_t ld_rows, hipStream_t stream)
{
    const int64_t vecs = (width + Vec<T>::n - 1) / Vec<T>::n;
    const Lay l = lay_out(vecs);
    const int64_t blocks = std::max<int64_t>(1, (r.tokens + r.tokens_per_block - 1) / r.tokens_per_block);
    const int64_t parts = std::max<int64_t>(1, std::min<int64_t>((vecs + l.tx - 1) / l.tx, 512 / blocks));
    hipLaunchKernelGGL(route_dispatch<T>, dim3((unsigned)blocks, (unsigned)parts), dim3(kThreads), 0, stream, r, static_cast<const T *>(x), (long)ld_x,
                       (int)width, l.tx, static_cast<T *>(rows), (long)ld_rows);
    return launched("route_dispatch launch");
}
template <typename T>
int run_dispatch_i8(const Route &r, const void *x, int64_t ld_x, int64_t width, int8_t *q, int64_t ld_q, float *scale, hipStream_t stream)
{
    const Lay l = lay_out((width + Vec<T>::n - 1) / Vec<T>::n);
    const int64_t blocks = std::max<int64_t>(1, (r.tokens + r.tokens_per_block - 1) / r.tokens_per_block);
    hipLaunchKernelGGL(route_dispatch_i8<T>, dim3((unsigned)blocks), dim3(kThreads), 0, stream, r, static_cast<const T *>(x), (long)ld_x, (int)width, l.tx,
                       q, (long)ld_q, scale);
    return launched("route_dispatch_i8 launch");
}
template <typename T>
int run_quantize(const void *x, int64_t ld_x, int64_t rows, int64_t width, int8_t *q, int64_t ld_q, float *scale, hipStream_t stream)
{
    const Lay l = lay_out((width + Vec<T>::n - 1) / Vec<T>::n);
    const int64_t blocks = (rows + l.ty - 1) / l.ty;
    hipLaunchKernelGGL(quantize_rows<T>, dim3((unsigned)blocks), dim3(kThreads), 0, stream, static_cast<const T *>(x), (long)ld_x, (long)rows, (int)width, l.tx,
                       q, (long)ld_q, scale);
    return launched("quantize_rows launch");
}
template <typename T>
int run_combine(const void *rows, int64_t ld_rows, const float *weight, const int32_t *row_of_slot, int64_t tokens, int k, int64_t width, void *y,
                int64_t ld_y, hipStream_t stream)
{
    const int64_t vecs = (width + Vec<T>::n - 1) / Vec<T>::n;
    const Lay l = lay_out(vecs);
    const int64_t blocks = (tokens + l.ty - 1) / l.ty;
    const int64_t parts = std::max<int64_t>(1, std::min<int64_t>((vecs + l.tx - 1) / l.tx, 1024 / blocks));
    hipLaunchKernelGGL(route_combine<T>, dim3((unsigned)blocks, (unsigned)parts), dim3(kThreads), 0, stream, static_cast<const T *>(rows), (long)ld_rows, weight,
                       row_of_slot, (long)tokens, k, (int)width, l.tx, static_cast<T *>(y), (long)ld_y);
    return launched("route_combine launch");
}
template <typename T>
int run_combine_grad(const void *dy, int64_t ld_dy, const void *rows, int64_t ld_rows, const float *weight, const int32_t *row_of_slot, const int32_t *held_at,
                     int64_t tokens, int k, int64_t width, void *drows, int64_t ld_drows, float *dweight, hipStream_t stream)
{
    const Lay l = lay_out((width + Vec<T>::n - 1) / Vec<T>::n);
    const int64_t blocks = (tokens + l.ty - 1) / l.ty;
    hipLaunchKernelGGL(route_combine_grad<T>, dim3((unsigned)blocks), dim3(kThreads), 0, stream, static_cast<const T *>(dy), (long)ld_dy, static_cast<const T *>(rows),
                       (long)ld_rows, weight, row_of_slot, held_at, (long)tokens, k, (int)width, l.tx, static_cast<T *>(drows), (long)ld_drows, dweight);
    return launched("route_combine_grad launch");
}

}  // namespace

#define BY_DTYPE(dtype, call, ...)                                          \
    ((dtype) == OPEVO_F32 ? call<float>(__VA_ARGS__)                        \
     : (dtype) == OPEVO_BF16 ? call<__bf16>(__VA_ARGS__) : call<_Float16>(__VA_ARGS__))

extern "C" int opevo_route_workspace(int64_t tokens, int k, int experts, size_t *bytes)
{
    if (!bytes) return fail(OPEVO_E_ARG, "route_workspace: bytes is NULL");
    if (int rc = check_route("route_workspace", tokens, k, experts)) return rc;
    const int64_t slots = tokens * k, chunk = chunk_of(slots, experts);
    *bytes = slots > kCountAlone ? sizeof(int) * (size_t)((slots + chunk - 1) / chunk) * experts : 0;
    return OPEVO_OK;
}

static int check_dispatch(const char *who, const int32_t *expert, int64_t tokens, int k, int experts, const void *x, int64_t ld_x, int dtype, int64_t width,
                          int32_t *offsets, int32_t *row_of_slot)
{
    if (int rc = check_route(who, tokens, k, experts)) return rc;
    if (!known(dtype)) return fail(OPEVO_E_ARG, "%s: unknown element type %d", who, dtype);
    if (int rc = check_words(who, "offsets", offsets)) return rc;
    if (tokens == 0) return OPEVO_OK;       // nothing else is read or written
    if (int rc = check_words(who, "expert", expert)) return rc;
    if (int rc = check_words(who, "row_of_slot", row_of_slot)) return rc;
    return check_rows(who, "x", x, ld_x, width, size_of(dtype));
}

extern "C" int opevo_route_dispatch(const int32_t *expert, int64_t tokens, int k, int experts, const void *x, int64_t ld_x, int dtype, int64_t width,
                                    int32_t *offsets, int32_t *row_of_slot, void *rows, int64_t ld_rows, void *workspace, size_t workspace_bytes, void *stream)
{
    const char *who = "route_dispatch";
    if (int rc = check_dispatch(who, expert, tokens, k, experts, x, ld_x, dtype, width, offsets, row_of_slot)) return rc;
    if (tokens > 0)
        if (int rc = check_rows(who, "rows", rows, ld_rows, width, size_of(dtype))) return rc;
    Route r;
    const hipStream_t on = static_cast<hipStream_t>(stream);
    if (int rc = plan_route(who, expert, tokens, k, experts, offsets, row_of_slot, workspace, workspace_bytes, on, &r)) return rc;
    return BY_DTYPE(dtype, run_dispatch, r, x, ld_x, width, rows, ld_rows, on);
}

extern "C" int opevo_route_dispatch_i8(const int32_t *expert, int64_t tokens, int k, int experts, const void *x, int64_t ld_x, int dtype, int64_t width,
                                       int32_t *offsets, int32_t *row_of_slot, int8_t *q, int64_t ld_q, float *scale, void *workspace, size_t workspace_bytes,
                                       void *stream)
{
    const char *who = "route_dispatch_i8";
    if (int rc = check_dispatch(who, expert, tokens, k, experts, x, ld_x, dtype, width, offsets, row_of_slot)) return rc;
    if (tokens > 0) {
        if (int rc = check_rows(who, "q", q, ld_q, width, 1)) return rc;
        if (int rc = check_words(who, "scale", scale)) return rc;
    }
    Route r;
    const hipStream_t on = static_cast<hipStream_t>(stream);
    if (int rc = plan_route(who, expert, tokens, k, experts, offsets, row_of_slot, workspace, workspace_bytes, on, &r)) return rc;
    return BY_DTYPE(dtype, run_dispatch_i8, r, x, ld_x, width, q, ld_q, scale, on);
}

extern "C" int opevo_quantize_rows_i8(const void *x, int64_t ld_x, int dtype, int64_t rows, int64_t width, int8_t *q, int64_t ld_q, float *scale, void *stream)
{
    const char *who = "quantize_rows_i8";
    if (!known(dtype)) return fail(OPEVO_E_ARG, "%s: unknown element type %d", who, dtype);
    if (rows < 0 || rows > INT32_MAX) return fail(OPEVO_E_ARG, "%s: %lld rows", who, (long long)rows);
    if (rows == 0) return OPEVO_OK;
    if (int rc = check_rows(who, "x", x, ld_x, width, size_of(dtype))) return rc;
    if (int rc = check_rows(who, "q", q, ld_q, width, 1)) return rc;
    if (int rc = check_words(who, "scale", scale)) return rc;
    return BY_DTYPE(dtype, run_quantize, x, ld_x, rows, width, q, ld_q, scale, static_cast<hipStream_t>(stream));
}

extern "C" int opevo_route_combine(const void *rows, int64_t ld_rows, int dtype, const float *weight, const int32_t *row_of_slot, int64_t tokens, int k,
                                   int64_t width, void *y, int64_t ld_y, void *stream)
{
    const char *who = "route_combine";
    if (int rc = check_route(who, tokens, k, 1)) return rc;
    if (!known(dtype)) return fail(OPEVO_E_ARG, "%s: unknown element type %d", who, dtype);
    if (tokens == 0) return OPEVO_OK;
    if (int rc = check_rows(who, "rows", rows, ld_rows, width, size_of(dtype))) return rc;
    if (int rc = check_rows(who, "y", y, ld_y, width, size_of(dtype))) return rc;
    if (int rc = check_words(who, "row_of_slot", row_of_slot)) return rc;
    if (weight)
        if (int rc = check_words(who, "weight", weight)) return rc;
    return BY_DTYPE(dtype, run_combine, rows, ld_rows, weight, row_of_slot, tokens, k, width, y, ld_y, static_cast<hipStream_t>(stream));
}

extern "C" int opevo_route_combine_grad(const void *dy, int64_t ld_dy, const void *rows, int64_t ld_rows, int dtype, const float *weight,
                                        const int32_t *row_of_slot, const int32_t *offsets, int experts, int64_t tokens, int k, int64_t width, void *drows,
                                        int64_t ld_drows, float *dweight, void *stream)
{
    const char *who = "route_combine_grad";
    if (int rc = check_route(who, tokens, k, experts)) return rc;
    if (!known(dtype)) return fail(OPEVO_E_ARG, "%s: unknown element type %d", who, dtype);
    if (tokens == 0) return OPEVO_OK;
    if (int rc = check_rows(who, "dy", dy, ld_dy, width, size_of(dtype))) return rc;
    if (int rc = check_rows(who, "rows", rows, ld_rows, width, size_of(dtype))) return rc;
    if (int rc = check_rows(who, "drows", drows, ld_drows, width, size_of(dtype))) return rc;
    if (int rc = check_words(who, "weight", weight)) return rc;
    if (int rc = check_words(who, "row_of_slot", row_of_slot)) return rc;
    if (int rc = check_words(who, "offsets", offsets)) return rc;
    if (int rc = check_words(who, "dweight", dweight)) return rc;
    return BY_DTYPE(dtype, run_combine_grad, dy, ld_dy, rows, ld_rows, weight, row_of_slot, offsets + experts, tokens, k, width, drows, ld_drows, dweight,
                    static_cast<hipStream_t>(stream));
}
