// Routing of an expert layer: tokens to the rows of their experts (dispatch), rows back to their tokens with weights
// (combine), the gradients of both, and rows of numbers to 8-bit integers with a scale each.
//
// T tokens have k slots each; slot s = t * k + j names an expert or none that is held here.  The stable sort of the slots by
// expert gives every held slot a row; everything else is rows copied or summed.  None of it has arithmetic to speak of: the
// floor is the bytes, and for a few tokens the launch.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdint>

#include "launch.hpp"
#include "narrow.hpp"
#include "wave.hpp"

namespace {

constexpr int kThreads = 256;
constexpr int kMaxExperts = OPEVO_ROUTE_MAX_EXPERTS;

// A launch has fewer than 2^32 threads along an extent of its grid: workgroups go on in the third.
constexpr int kGridX = 1 << 23;
__device__ __forceinline__ long this_block() { return (long)blockIdx.z * kGridX + blockIdx.x; }
dim3 spread(int64_t blocks, int64_t parts = 1)
{
    return dim3((unsigned)std::min<int64_t>(blocks, kGridX), (unsigned)parts, (unsigned)((blocks + kGridX - 1) / kGridX));
}

// A row is taken in pieces of 16 bytes.  Rows start wherever the caller's row length puts them, so all accesses are made for any alignment (the hardware's
// 16-byte loads and stores take any address; the compiler is told nothing more).  Where the width is no multiple of a piece, the last piece ends with the row and overlaps the
// one before it: both write the same values.  A row shorter than a piece is one, taken element by element.
template <typename T> struct Vec {
    static constexpr int n = 16 / sizeof(T);
    T v[n];
};
template <typename T, bool WIDE> struct Pieces {     // WIDE: rows of at least a piece
    int width, count;
    __device__ explicit Pieces(int w) : width(w), count((w + Vec<T>::n - 1) / Vec<T>::n) {}
    __device__ __forceinline__ int first(int i) const { return WIDE ? min(i * Vec<T>::n, width - Vec<T>::n) : 0; }
    // how many of its elements the piece before has too
    __device__ __forceinline__ int twice(int i) const { return WIDE ? i * Vec<T>::n - first(i) : 0; }
    __device__ __forceinline__ Vec<T> load(const T *row, int i) const
    {
        Vec<T> r = {};
        if (WIDE) __builtin_memcpy(&r, row + first(i), 16);
        else
#pragma unroll
            for (int e = 0; e < Vec<T>::n; ++e)
                if (e < width) r.v[e] = row[e];
        return r;
    }
    template <typename O> __device__ __forceinline__ void store(O *row, int i, const O (&v)[Vec<T>::n]) const
    {
        if (WIDE) __builtin_memcpy(row + first(i), v, sizeof v);
        else
#pragma unroll
            for (int e = 0; e < Vec<T>::n; ++e)
                if (e < width) row[e] = v[e];
    }
};

// ------------------------------------------------------------------ the sort
// How many slots of a chunk go to each expert: counts[chunk][expert].
__global__ __launch_bounds__(kThreads)
void route_count(const int *__restrict__ expert, long slots, int chunk, int experts, int *__restrict__ counts)
{
    __shared__ int hist[kMaxExperts];
    const long first = (long)blockIdx.x * chunk, last = first + chunk < slots ? first + chunk : slots;
    for (long s0 = first; s0 < last; s0 += kThreads * 4) {
        unsigned e[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) e[u] = s0 + u * kThreads + threadIdx.x < last ? (unsigned)expert[s0 + u * kThreads + threadIdx.x] : ~0u;
        if (s0 == first) {                  // while the first ones come
            for (int i = threadIdx.x; i < experts; i += kThreads) hist[i] = 0;
            __syncthreads();
        }
#pragma unroll
        for (int u = 0; u < 4; ++u)
            if (e[u] < (unsigned)experts) atomicAdd(&hist[e[u]], 1);
    }
    __syncthreads();
    for (int e = threadIdx.x; e < experts; e += kThreads) counts[(long)blockIdx.x * experts + e] = hist[e];
}

// The counts of a chunk become those of all chunks before it, and behind the last chunk come those of all: a workgroup of the dispatch reads two lines of them instead of all
// lines, which would make the sort's work grow with the square of the slots.  A workgroup takes kScanCols experts; each of its lines of lanes takes as many chunks as the others,
// adds them up, and goes through them again from the sum of the lines before it.
constexpr int kScanCols = 16, kScanThreads = 1024, kScanLines = kScanThreads / kScanCols;
__global__ __launch_bounds__(kScanThreads)
void route_scan(int *counts, int chunks, int experts)
{
    __shared__ int sums[kScanLines][kScanCols];
    const int col = (int)threadIdx.x % kScanCols, line = (int)threadIdx.x / kScanCols, e = blockIdx.x * kScanCols + col;
    const int share = (chunks + kScanLines - 1) / kScanLines, first = min(line * share, chunks), last = min(first + share, chunks);
    const bool on = e < experts;
    int sum = 0;
    if (on)
#pragma unroll 8
        for (int c = first; c < last; ++c) sum += counts[(long)c * experts + e];
    sums[line][col] = sum;
    __syncthreads();
    if (!on) return;
    int run = 0;
    for (int l = 0; l < line; ++l) run += sums[l][col];
#pragma unroll 8
    for (int c = first; c < last; ++c) {
        const int n = counts[(long)c * experts + e];
        counts[(long)c * experts + e] = run;
        run += n;
    }
    if (line == kScanLines - 1) counts[(long)chunks * experts + e] = run;
}

constexpr int kFew = 16;                // slots that one wave sorts by comparing them
constexpr int kOwn = 64;                // slots of a workgroup at most: one wave ranks them

struct Route {
    const int *expert;
    long tokens;
    int k, experts;
    const int *counts;      // NULL: every workgroup counts all slots itself
    int chunk, chunks;
    bool scanned;           // counts[c] are those of the chunks before c, c up to `chunks`
    int tokens_per_block;
    long blocks;
    int *offsets, *row_of_slot;
};
struct Sorted { __attribute__((aligned(16))) int total[kMaxExperts]; int before[kMaxExperts], place[kOwn], held; };

// Rows of this workgroup's slots into place[] (-1: none), from the slots' experts alone: a slot's row is the number of slots of
// lower experts, plus the earlier slots of its own.  Earlier slots are those of earlier chunks (counted by route_count; a column sum, which route_scan has made of it where there are many), those of
// its chunk before this workgroup's first (counted here), and those of this workgroup before it.  Integer counts: any order gives the same.
// held: the number of slots that have a row.
__device__ __forceinline__ void route_rows(const Route &r, long first_slot, int own, Sorted &s, bool writes)
{
    const int tid = threadIdx.x;
    // A few slots (one token: 2.5 us instead of 3.1; 64 slots take 4.7 this way and 3.6 the other): a lane for each, whose row is the number of smaller keys, a key being the
    // expert and the slot.
    if (r.tokens * r.k <= kFew) {
        if (tid < 64) {
            const int slots = (int)(r.tokens * r.k), e = tid < slots ? r.expert[tid] : -1;
            const bool valid = (unsigned)e < (unsigned)r.experts;
            const int key = valid ? e * 64 + tid : INT32_MAX;
            s.total[tid] = key;
            exchange();
            auto smaller = [&](int than) {
                int n = 0;
                for (int i = 0; i < slots; i += 4)          // one wave, whose LDS accesses keep their order
#pragma unroll
                    for (int u = 0; u < 4; ++u) n += s.total[i + u] < than;
                return n;
            };
            const int at = tid - (int)first_slot, row = smaller(key), held = __popcll(__ballot(valid));
            if (at >= 0 && at < own) s.place[at] = valid ? row : -1;
            if (tid == 0) s.held = held;
            if (writes)
                for (int i = tid; i <= r.experts; i += 64) r.offsets[i] = smaller(i * 64);
        }
        __syncthreads();
        return;
    }
    const int slot = tid < own ? r.expert[first_slot + tid] : -1;
    for (int e = tid; e < r.experts; e += kThreads) s.total[e] = s.before[e] = 0;
    __syncthreads();
    if (r.counts) {
        const int at = (int)(first_slot >> __builtin_ctz(r.chunk));     // chunks are powers of two
        if (r.scanned)
            for (int e = tid; e < r.experts; e += kThreads) {
                s.total[e] = r.counts[(long)r.chunks * r.experts + e];
                atomicAdd(&s.before[e], r.counts[(long)at * r.experts + e]);
            }
        const int lines = kThreads / r.experts > 1 ? kThreads / r.experts : 1, line = lines > 1 ? tid / r.experts : 0;
        for (int e = lines > 1 ? tid - line * r.experts : tid; !r.scanned && e < r.experts && line < lines; e += kThreads) {
            int total = 0, before = 0;
#pragma unroll 16
            for (int c = line; c < r.chunks; c += lines) {
                const int n = r.counts[c * r.experts + e];
                total += n;
                before += c < at ? n : 0;
            }
            atomicAdd(&s.total[e], total);
            atomicAdd(&s.before[e], before);
        }
        for (long i0 = (long)at * r.chunk; i0 < first_slot; i0 += kThreads * 4) {
            unsigned e[4];
#pragma unroll
            for (int u = 0; u < 4; ++u) e[u] = i0 + u * kThreads + tid < first_slot ? (unsigned)r.expert[i0 + u * kThreads + tid] : ~0u;
#pragma unroll
            for (int u = 0; u < 4; ++u)
                if (e[u] < (unsigned)r.experts) atomicAdd(&s.before[e[u]], 1);
        }
    } else {
        // both counts in one word, neither beyond 16 bits (kCountAlone slots at most)
        const int slots = (int)(r.tokens * r.k);
        for (int i0 = 0; i0 < slots; i0 += kThreads * 4) {
            unsigned e[4];
#pragma unroll
            for (int u = 0; u < 4; ++u) e[u] = i0 + u * kThreads + tid < slots ? (unsigned)r.expert[i0 + u * kThreads + tid] : ~0u;
#pragma unroll
            for (int u = 0; u < 4; ++u)
                if (e[u] < (unsigned)r.experts) atomicAdd(&s.total[e[u]], i0 + u * kThreads + tid < first_slot ? 0x10001 : 1);
        }
    }
    __syncthreads();
    if (tid < 64) {                         // exclusive sums over the experts, 64 at a time, by the wave that has the slots
        int run = 0;
        for (int e0 = 0; e0 < r.experts; e0 += 64) {
            const int e = e0 + tid, word = e < r.experts ? s.total[e] : 0, n = r.counts ? word : word & 0xffff;
            int sum = n;
#pragma unroll
            for (int o = 1; o < 64; o <<= 1) {
                const int up = __shfl_up(sum, o);
                if (tid >= o) sum += up;
            }
            if (e < r.experts) {
                s.before[e] = (r.counts ? s.before[e] : word >> 16) + run + sum - n;
                if (writes) r.offsets[e] = run + sum - n;
            }
            run += __shfl(sum, 63);
        }
        if (tid == 0) {
            s.held = run;
            if (writes) r.offsets[r.experts] = run;
        }
        exchange();
        int earlier = 0;
        for (int i = 0; i < own; ++i) {
            const int other = __builtin_amdgcn_readlane(slot, i);
            earlier += i < tid && other == slot;
        }
        if (tid < own) s.place[tid] = (unsigned)slot < (unsigned)r.experts ? s.before[slot] + earlier : -1;
    }
    __syncthreads();
}

struct Lay { int tx, ty, hold; };
// `tx` lanes (a power of two) side by side on a row of `pieces`, `hold` pieces each, the others on further rows.  One piece a lane is the shortest way through a row; where there
// are more rows than the chip holds at once, more pieces a lane keep more bytes on their way and leave a row to fewer waves.
static Lay lay_out(int64_t pieces, int64_t rows, int most)
{
    int tx = 1, hold = 1;
    while (tx < kThreads && tx < pieces) tx *= 2;
    const auto many = [&] { return tx > 64 && rows * (tx / 2) / 64 >= 4096; };      // a wave to a row at least: its accesses stay whole lines
    while (hold < most && (tx * hold < pieces || many())) {
        if (many() && tx * hold >= pieces) tx /= 2;
        hold *= 2;
    }
    return {tx, kThreads / tx, hold};
}

// ------------------------------------------------------------------ dispatch
// Bound by memory: 16384 tokens of 4096 bf16 to two rows each move 403 MB in 83 us behind the count's 4.7 (4.6 TB/s in all; a large copy 5.15).  A token is read once and written k times; the first pieces are on their way while the slots
// are sorted, the next ones while a piece is written.
template <typename T, int kHold, bool WIDE>
__global__ __launch_bounds__(kThreads)
void route_dispatch(Route r, const T *__restrict__ x, long ld_x, int width, int tx, T *__restrict__ rows, long ld_rows)
{
    __shared__ Sorted s;
    const long block = this_block(), first = block * r.tokens_per_block;
    if (first >= r.tokens && block > 0) return;
    const int tokens = (int)(r.tokens - first < r.tokens_per_block ? r.tokens - first : r.tokens_per_block), own = tokens * r.k;
    const Pieces<T, WIDE> at(width);
    const int lane = (int)threadIdx.x & (tx - 1), ty = kThreads >> __builtin_ctz(tx), line = (int)threadIdx.x >> __builtin_ctz(tx);
    const int step = tx * gridDim.y * kHold, start = blockIdx.y * tx * kHold + lane;
    Vec<T> v[kHold], w[kHold];
    auto load = [&](Vec<T> (&to)[kHold], int t, int c) {
#pragma unroll
        for (int u = 0; u < kHold; ++u)
            if (t < tokens && c + u * tx < at.count) to[u] = at.load(x + (first + t) * ld_x, c + u * tx);
    };
    int t = line, c = start;
    load(v, t, c);
    route_rows(r, first * r.k, own, s, block == 0 && blockIdx.y == 0);
    if (blockIdx.y == 0 && (int)threadIdx.x < own) r.row_of_slot[first * r.k + threadIdx.x] = s.place[threadIdx.x];
    while (t < tokens) {
        int next_t = t, next_c = c + step;
        if (next_c >= at.count) { next_t += ty; next_c = start; }
        load(w, next_t, next_c);
        for (int j = 0; j < r.k; ++j) {
            const int row = s.place[t * r.k + j];
            if (row < 0) continue;
#pragma unroll
            for (int u = 0; u < kHold; ++u)
                if (c + u * tx < at.count) at.store(rows + row * ld_rows, c + u * tx, v[u].v);
        }
#pragma unroll
        for (int u = 0; u < kHold; ++u) v[u] = w[u];
        t = next_t; c = next_c;
    }
    // rows that no slot goes to
    const Vec<T> zero = {};
    for (long row = s.held + block * ty + line; row < r.tokens * r.k; row += r.blocks * ty)
        for (int i = blockIdx.y * tx + lane; i < at.count; i += tx * gridDim.y) at.store(rows + row * ld_rows, i, zero.v);
}

// ------------------------------------------------------------------ rows to 8 bits
// Magnitudes as bits without the sign: their order is that of the values, and infinities and NaNs come last.
typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));
__device__ __forceinline__ unsigned magnitude(const Vec<float> &v)
{
    unsigned m = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) m = max(m, __float_as_uint(v.v[i]) & 0x7fffffffu);
    return m;
}
template <typename T> __device__ __forceinline__ unsigned magnitude(const Vec<T> &v)
{
    unsigned w[4];
    __builtin_memcpy(w, v.v, 16);
    u16x2 m = {0, 0};
#pragma unroll
    for (int i = 0; i < 4; ++i) m = __builtin_elementwise_max(m, __builtin_bit_cast(u16x2, w[i] & 0x7fff7fffu));
    return max(m.x, m.y);
}
template <typename T> __device__ __forceinline__ float value_of(unsigned m) { return (float)__builtin_bit_cast(T, (unsigned short)m); }
template <> __device__ __forceinline__ float value_of<float>(unsigned m) { return __uint_as_float(m); }

// q = round(127 x / a), a the row's largest magnitude.  With 127 x computed first (exact for 16-bit inputs: 11 + 7 bits) and one
// division, the quotient of two numbers of at most 18 and 11 bits is a tie in fp32 only where it is one exactly, so the result is the
// rounding of the exact quotient; of fp32 inputs 127 x is rounded too, and where the exact quotient is within 2^-23 of its value from a tie (1.52e-5 at
// the most) the other integer may come out.  8192 rows of 4096 bf16 take 25 us (4.0 TB/s).  A division takes ten instructions: x times 127 / a, off by at most
// 2.3e-5 from that, rounds to the same integer unless it is within 4e-5 of a tie, and only then are the piece's eight values divided.
template <typename T> struct Quantizer {
    float a, pre, inv, scale;
    bool on, plain;
    __device__ explicit Quantizer(unsigned m)
    {
        const float largest = value_of<T>(m);
        const bool finite = largest < __uint_as_float(0x7f800000u);
        pre = largest > 1e30f ? 0x1p-7f : largest < 1e-30f ? 0x1p96f : 1.f;      // neither 127 x nor 127 / a overflows
        a = largest * pre;
        inv = 127.f / a;
        on = finite && m > 0;
        plain = pre == 1.f;
        scale = finite ? largest / 127.f : __uint_as_float(0x7fc00000u);
    }
    __device__ __forceinline__ void operator()(const Vec<T> &x, int8_t (&q)[Vec<T>::n]) const
    {
        constexpr float kRound = 12582912.f;                // 1.5 * 2^23: what is added to it is rounded to an integer, in its low bits
        unsigned word[Vec<T>::n];
        float off = plain ? 0.f : 1.f;
#pragma unroll
        for (int i = 0; i < Vec<T>::n; ++i) {
            const float v = (float)x.v[i], r = fmaf(v, inv, kRound);
            off = fmaxf(off, fabsf(fmaf(v, inv, kRound - r)));
            word[i] = __float_as_uint(r);
        }
        if (off > 0.49996f)
#pragma unroll
            for (int i = 0; i < Vec<T>::n; ++i) word[i] = __float_as_uint(127.f * ((float)x.v[i] * pre) / a + kRound);
        unsigned packed[Vec<T>::n / 4];
#pragma unroll
        for (int i = 0; i < Vec<T>::n / 4; ++i) {
            const unsigned lo = __builtin_amdgcn_perm(word[4 * i + 1], word[4 * i], 0x0c0c0400u), hi = __builtin_amdgcn_perm(word[4 * i + 3], word[4 * i + 2], 0x04000c0cu);
            packed[i] = on ? lo | hi : 0u;
        }
        __builtin_memcpy(q, packed, sizeof packed);
    }
};

// The maximum over the tx lanes of a row (red: one word a wave).  tx > 64: for all threads of the workgroup together.
__device__ __forceinline__ unsigned row_max(unsigned m, int tx, unsigned *red)
{
    for (int o = 1; o < tx && o < 64; o <<= 1) m = max(m, (unsigned)__shfl_xor((int)m, o));
    if (tx > 64) {
        __syncthreads();
        if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = m;
        __syncthreads();
        const int w0 = (threadIdx.x >> __builtin_ctz(tx)) * (tx / 64);
        for (int w = 0; w < tx / 64; ++w) m = max(m, red[w0 + w]);
    }
    return m;
}

// A row's pieces in registers, as many as a lane holds; rows longer than that are read a second time for the pieces beyond.
template <typename T, int HOLD, bool WIDE> struct Held {
    Vec<T> v[HOLD];
    unsigned m;
    __device__ __forceinline__ void load(const Pieces<T, WIDE> &at, const T *row, int lane, int tx, bool on)
    {
#pragma unroll
        for (int u = 0; u < HOLD; ++u) {
            v[u] = {};
            if (on && lane + u * tx < at.count) v[u] = at.load(row, lane + u * tx);
        }
    }
    __device__ __forceinline__ void scan(const Pieces<T, WIDE> &at, const T *row, int lane, int tx, bool on)
    {
        m = 0;
#pragma unroll
        for (int u = 0; u < HOLD; ++u) m = max(m, magnitude(v[u]));
        if (on)
            for (int i = lane + HOLD * tx; i < at.count; i += tx) m = max(m, magnitude(at.load(row, i)));
    }
    template <typename F> __device__ __forceinline__ void each(const Pieces<T, WIDE> &at, const T *row, int lane, int tx, F &&f) const
    {
#pragma unroll
        for (int u = 0; u < HOLD; ++u)
            if (lane + u * tx < at.count) f(lane + u * tx, v[u]);
        for (int i = lane + HOLD * tx; i < at.count; i += tx) f(i, at.load(row, i));
    }
};

template <typename T, int kHold, bool WIDE>
__global__ __launch_bounds__(kThreads)
void quantize_rows(const T *__restrict__ x, long ld_x, long rows, int width, int tx, int8_t *__restrict__ q, long ld_q, float *__restrict__ scale)
{
    __shared__ unsigned red[kThreads / 64];
    const int lane = (int)threadIdx.x & (tx - 1), ty = kThreads >> __builtin_ctz(tx);
    const long row = this_block() * ty + ((int)threadIdx.x >> __builtin_ctz(tx));
    const bool on = row < rows;
    const T *src = x + (on ? row : 0) * ld_x;
    const Pieces<T, WIDE> at(width);
    Held<T, kHold, WIDE> h;
    h.load(at, src, lane, tx, on);
    h.scan(at, src, lane, tx, on);
    const unsigned m = row_max(h.m, tx, red);
    if (!on) return;
    const Quantizer<T> z(m);
    h.each(at, src, lane, tx, [&](int i, const Vec<T> &v) {
        int8_t out[Vec<T>::n];
        z(v, out);
        at.store(q + row * ld_q, i, out);
    });
    if (lane == 0) scale[row] = z.scale;
}

template <typename T, int kHold, bool WIDE>
__global__ __launch_bounds__(kThreads)
void route_dispatch_i8(Route r, const T *__restrict__ x, long ld_x, int width, int tx, int8_t *__restrict__ q, long ld_q, float *__restrict__ scale)
{
    __shared__ Sorted s;
    __shared__ unsigned red[kThreads / 64];
    const long block = this_block(), first = block * r.tokens_per_block;
    if (first >= r.tokens && block > 0) return;
    const int tokens = (int)(r.tokens - first < r.tokens_per_block ? r.tokens - first : r.tokens_per_block), own = tokens * r.k;
    const int lane = (int)threadIdx.x & (tx - 1), ty = kThreads >> __builtin_ctz(tx), line = (int)threadIdx.x >> __builtin_ctz(tx);
    const Pieces<T, WIDE> at(width);
    Held<T, kHold, WIDE> h, next;
    h.load(at, x + (first + line) * ld_x, lane, tx, line < tokens);
    route_rows(r, first * r.k, own, s, block == 0);
    if ((int)threadIdx.x < own) r.row_of_slot[first * r.k + threadIdx.x] = s.place[threadIdx.x];
    for (int t0 = 0; t0 < tokens; t0 += ty) {               // alike for all threads: row_max is for all together
        const int t = t0 + line;
        const bool on = t < tokens;
        const T *src = x + (first + t) * ld_x;
        next.load(at, src + ty * ld_x, lane, tx, t + ty < tokens);
        h.scan(at, src, lane, tx, on);
        const unsigned m = row_max(h.m, tx, red);
        if (on) {
            const Quantizer<T> z(m);
            h.each(at, src, lane, tx, [&](int i, const Vec<T> &v) {
                int8_t out[Vec<T>::n];
                z(v, out);
                for (int j = 0; j < r.k; ++j) {
                    const int row = s.place[t * r.k + j];
                    if (row >= 0) at.store(q + row * ld_q, i, out);
                }
            });
            for (int j = lane; j < r.k; j += tx) {
                const int row = s.place[t * r.k + j];
                if (row >= 0) scale[row] = z.scale;
            }
        }
        h = next;
    }
    const int8_t zero[Vec<T>::n] = {};
    for (long row = s.held + block * ty + line; row < r.tokens * r.k; row += r.blocks * ty) {
        for (int i = lane; i < at.count; i += tx) at.store(q + row * ld_q, i, zero);
        if (lane == 0) scale[row] = 0.f;
    }
}

// ------------------------------------------------------------------ combine
// y[t] = sum_j w[t, j] rows[row_of_slot[t, j]], j ascending, in fp32, rounded once; a slot without a row adds nothing, whatever its weight.  Bound by memory: the rows
// of J slots are on their way together (8192 tokens, 4 slots, 4096 bf16: 339 MB in 70 - 78 us; J = 8 takes registers that more waves use better: 86).
constexpr int kSlots = 4;               // J

template <typename T, bool WIDE>
__global__ __launch_bounds__(kThreads)
void route_combine(const T *__restrict__ rows, long ld_rows, const float *__restrict__ weight, const int *__restrict__ row_of_slot,
                   long tokens, int k, int width, int tx, T *__restrict__ y, long ld_y)
{
    const int lane = (int)threadIdx.x & (tx - 1), ty = kThreads >> __builtin_ctz(tx);
    const long t = this_block() * ty + ((int)threadIdx.x >> __builtin_ctz(tx)), slots = tokens * k;
    if (t >= tokens) return;
    const Pieces<T, WIDE> at(width);
    for (int i = blockIdx.y * tx + lane; i < at.count; i += tx * gridDim.y) {
        float sum[Vec<T>::n] = {};
        for (int j0 = 0; j0 < k; j0 += kSlots) {
            // all places before the first row: loads return in order, and a place behind a row would be waited for with it
            int row[kSlots];
            float w[kSlots];
#pragma unroll
            for (int j = 0; j < kSlots; ++j) {
                const long slot = t * k + min(j0 + j, k - 1);
                row[j] = row_of_slot[slot];
                w[j] = weight ? weight[slot] : 1.f;
            }
            Vec<T> v[kSlots];
#pragma unroll
            for (int j = 0; j < kSlots; ++j) {
                if (j0 + j >= k || (unsigned)row[j] >= (unsigned long)slots) row[j] = -1;
                if (row[j] >= 0) v[j] = at.load(rows + row[j] * ld_rows, i);
            }
#pragma unroll
            for (int j = 0; j < kSlots; ++j)
                if (row[j] >= 0)
#pragma unroll
                    for (int e = 0; e < Vec<T>::n; ++e) sum[e] = fmaf(w[j], (float)v[j].v[e], sum[e]);
        }
        Vec<T> out;
#pragma unroll
        for (int e = 0; e < Vec<T>::n; ++e) out.v[e] = narrow<T>(sum[e]);
        at.store(y + t * ld_y, i, out.v);
    }
}

// drows[row_of_slot[s]] = w[s] dy[s / k], dw[s] = <dy[s / k], rows[row_of_slot[s]]>; rows from offsets[experts] on get zeros, slots without a row dw = 0.
// Bound by memory: 8192 tokens of 4096 bf16 with four rows each, 604 MB were each value moved once, take 118 us.  One row is read and one written at a time by as many waves as
// fit.  dy, which each slot reads again, mostly comes from beyond the L2s again: 506 MB are read there instead of 336, 775 in all (6.6 TB/s, some of it from the memory's own
// cache).  (All slots' rows at once, dy's pieces and the next row's held in registers: 140 - 180 us instead of 127 for that size.)
template <typename T, bool WIDE>
__global__ __launch_bounds__(kThreads)
void route_combine_grad(const T *__restrict__ dy, long ld_dy, const T *__restrict__ rows, long ld_rows, const float *__restrict__ weight,
                        const int *__restrict__ row_of_slot, const int *__restrict__ held_at, long tokens, int k, int width, int tx,
                        int share /* slots of a token a workgroup takes */, T *__restrict__ drows, long ld_drows, float *__restrict__ dweight)
{
    __shared__ float red[OPEVO_ROUTE_MAX_SLOTS][kThreads / 64];
    const int j0 = blockIdx.y * share, j1 = min(k, j0 + share);
    const int lane = (int)threadIdx.x & (tx - 1), ty = kThreads >> __builtin_ctz(tx), line = (int)threadIdx.x >> __builtin_ctz(tx);
    const long t = this_block() * ty + line, slots = tokens * k;
    const bool on = t < tokens;
    const Pieces<T, WIDE> at(width);
    for (int j = j0; j < j1; ++j) {
        const int row = on ? row_of_slot[t * k + j] : -1;
        float dot = 0.f;
        if ((unsigned)row < (unsigned long)slots) {
            const float w = weight[t * k + j];
            for (int i = lane; i < at.count; i += tx) {
                const Vec<T> g = at.load(dy + t * ld_dy, i), v = at.load(rows + row * ld_rows, i);
                const int twice = at.twice(i);
                if (twice == 0)
#pragma unroll
                    for (int e = 0; e < Vec<T>::n; ++e) dot = fmaf((float)g.v[e], (float)v.v[e], dot);
                else
                    for (int e = 0; e < Vec<T>::n; ++e)
                        if (e >= twice) dot = fmaf((float)g.v[e], (float)v.v[e], dot);
                Vec<T> out;
#pragma unroll
                for (int e = 0; e < Vec<T>::n; ++e) out.v[e] = narrow<T>(w * (float)g.v[e]);
                at.store(drows + row * ld_drows, i, out.v);
            }
        }
        for (int o = 1; o < tx && o < 64; o <<= 1) dot += __shfl_xor(dot, o);
        if (tx <= 64) {
            if (on && lane == 0) dweight[t * k + j] = dot;
        } else if ((threadIdx.x & 63) == 0) {
            red[j][threadIdx.x >> 6] = dot;
        }
    }
    if (tx > 64) {
        __syncthreads();
        for (int j = j0 + lane; on && j < j1; j += tx) {
            float dot = 0.f;
            for (int i = 0; i < tx / 64; ++i) dot += red[j][line * (tx / 64) + i];
            dweight[t * k + j] = dot;
        }
    }
    const Vec<T> zero = {};
    const int held = *held_at;
    for (long row = (held > 0 ? held : 0) + ((long)blockIdx.y * gridDim.x * gridDim.z + this_block()) * ty + line; row < slots; row += (long)gridDim.y * gridDim.x * gridDim.z * ty)
        for (int i = lane; i < at.count; i += tx) at.store(drows + row * ld_drows, i, zero.v);
}

// ------------------------------------------------------------------ host side
using opevo::fail;
using opevo::launch;

bool aligned(const void *p, size_t to) { return reinterpret_cast<uintptr_t>(p) % to == 0; }
size_t size_of(int dtype) { return dtype == OPEVO_F32 ? 4 : 2; }
bool known(int dtype) { return dtype == OPEVO_F32 || dtype == OPEVO_BF16 || dtype == OPEVO_F16; }

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

// Up to this many slots every workgroup counts them all itself; beyond, route_count does it chunk by chunk.  Rows of 1024 bf16, two slots a token, 8 / 64 / 256 experts, us by
// themselves against counted: 2048 slots 4.8 / 4.7 / 5.7 against 6.7 / 6.9 / 9.3, 4096 6.9 / 6.9 / 7.9 against 8.0 / 8.5 / 10.4, 8192 10.6 / 10.7 / 11.6 against 9.6 / 11.6 / 11.4,
// 16384 20.7 / 20.7 / 21.3 against 13.2 / 15.0 / 14.4.
constexpr int64_t kCountAlone = 4096;
// A workgroup reads chunks * experts counts and half a chunk of slots on average.
int64_t chunk_of(int64_t slots, int experts)
{
    int64_t chunk = 256;
    while (chunk < 8192 && 8 * chunk * chunk < slots * experts) chunk *= 2;
    return chunk;
}

// Whether a third kernel adds the counts up along the chunks, or every workgroup (at most kOwn slots) does for itself: by what all of them together would read.  Rows
// of 64 bf16, us without / with the scan: 131072 slots of 128 experts (64 chunks) 21.6 / 20.7, 32768 of 1024 (16) 17.8 / 18.9, 131072 of 1024 (32) 41.8 / 33.8, 2^20 of 256 (128)
// 186 / 115, 2^23 of 256 (1024) 7250 / 880; rows of 2048, 2^20 slots of 256 experts 984 / 982.
bool scans(int64_t slots, int64_t chunks, int experts) { return slots * chunks * experts > (int64_t)1 << 30; }
size_t workspace_of(int64_t slots, int experts)
{
    if (slots <= kCountAlone) return 0;
    const int64_t chunk = chunk_of(slots, experts), chunks = (slots + chunk - 1) / chunk;
    return sizeof(int) * (size_t)(chunks + scans(slots, chunks, experts)) * experts;
}

// Fills r and, where it takes them, launches the count and the scan.
int plan_route(const char *who, const int32_t *expert, int64_t tokens, int k, int experts, int32_t *offsets, int32_t *row_of_slot,
               void *workspace, size_t workspace_bytes, hipStream_t stream, Route *r)
{
    const int64_t slots = tokens * k;
    r->expert = expert; r->tokens = tokens; r->k = k; r->experts = experts;
    r->counts = nullptr; r->chunk = 1; r->chunks = 0; r->scanned = false;
    r->offsets = offsets; r->row_of_slot = row_of_slot;
    if (slots > kCountAlone) {
        r->chunk = (int)chunk_of(slots, experts);
        r->chunks = (int)((slots + r->chunk - 1) / r->chunk);
        r->scanned = scans(slots, r->chunks, experts);
        const size_t need = workspace_of(slots, experts);
        if (!workspace || !aligned(workspace, 4) || workspace_bytes < need)
            return fail(OPEVO_E_ARG, "%s: the workspace holds %zu bytes of the %zu it takes, or is not aligned to 4 bytes", who, workspace ? workspace_bytes : 0, need);
        if (int rc = launch("route_count launch", route_count, dim3(r->chunks), dim3(kThreads), stream, expert, (long)slots, r->chunk, experts, static_cast<int *>(workspace))) return rc;
        if (r->scanned)
            if (int rc = launch("route_scan launch", route_scan, dim3((experts + kScanCols - 1) / kScanCols), dim3(kScanThreads), stream, static_cast<int *>(workspace), r->chunks, experts)) return rc;
        r->counts = static_cast<const int *>(workspace);
    }
    return OPEVO_OK;
}

// As many tokens a workgroup as leave 1024 workgroups, or one for each compute unit where every one counts all slots, in whole rounds of `ty`, but no more slots than a wave ranks.
void deal(Route *r, int ty)
{
    const int64_t most = kOwn / r->k, share = r->tokens / (r->counts ? 1024 : 256);
    r->tokens_per_block = (int)std::max<int64_t>(1, std::min(std::max<int64_t>(ty, share / ty * ty), most));
    r->blocks = std::max<int64_t>(1, (r->tokens + r->tokens_per_block - 1) / r->tokens_per_block);
}

template <typename T>
int run_dispatch(Route r, const void *x, int64_t ld_x, int64_t width, void *rows, int64_t ld_rows, hipStream_t stream)
{
    const int64_t pieces = (width + Vec<T>::n - 1) / Vec<T>::n;
    const Lay l = lay_out(pieces, r.tokens, 4);
    deal(&r, l.ty);
    const int64_t parts = std::max<int64_t>(1, std::min<int64_t>((pieces + l.tx * l.hold - 1) / (l.tx * l.hold), 512 / r.blocks));
    auto *k = width < Vec<T>::n ? route_dispatch<T, 1, false> : l.hold == 1 ? route_dispatch<T, 1, true> : l.hold == 2 ? route_dispatch<T, 2, true> : route_dispatch<T, 4, true>;
    return launch("route_dispatch launch", k, spread(r.blocks, parts), dim3(kThreads), stream, r, static_cast<const T *>(x), (long)ld_x,
                       (int)width, l.tx, static_cast<T *>(rows), (long)ld_rows);
}
template <typename T>
int run_dispatch_i8(Route r, const void *x, int64_t ld_x, int64_t width, int8_t *q, int64_t ld_q, float *scale, hipStream_t stream)
{
    const Lay l = lay_out((width + Vec<T>::n - 1) / Vec<T>::n, r.tokens, 4);
    deal(&r, l.ty);
    auto *k = width < Vec<T>::n ? route_dispatch_i8<T, 1, false> : l.hold == 1 ? route_dispatch_i8<T, 1, true> : l.hold == 2 ? route_dispatch_i8<T, 2, true> : route_dispatch_i8<T, 4, true>;
    return launch("route_dispatch_i8 launch", k, spread(r.blocks), dim3(kThreads), stream, r, static_cast<const T *>(x), (long)ld_x, (int)width, l.tx,
                       q, (long)ld_q, scale);
}
template <typename T>
int run_quantize(const void *x, int64_t ld_x, int64_t rows, int64_t width, int8_t *q, int64_t ld_q, float *scale, hipStream_t stream)
{
    const Lay l = lay_out((width + Vec<T>::n - 1) / Vec<T>::n, rows, 4);
    const int64_t blocks = (rows + l.ty - 1) / l.ty;
    auto *k = width < Vec<T>::n ? quantize_rows<T, 1, false> : l.hold == 1 ? quantize_rows<T, 1, true> : l.hold == 2 ? quantize_rows<T, 2, true> : quantize_rows<T, 4, true>;
    return launch("quantize_rows launch", k, spread(blocks), dim3(kThreads), stream, static_cast<const T *>(x), (long)ld_x, (long)rows, (int)width, l.tx,
                       q, (long)ld_q, scale);
}
template <typename T>
int run_combine(const void *rows, int64_t ld_rows, const float *weight, const int32_t *row_of_slot, int64_t tokens, int k, int64_t width, void *y,
                int64_t ld_y, hipStream_t stream)
{
    const int64_t pieces = (width + Vec<T>::n - 1) / Vec<T>::n;
    const Lay l = lay_out(pieces, tokens, 1);
    const int64_t blocks = (tokens + l.ty - 1) / l.ty;
    const int64_t parts = std::max<int64_t>(1, std::min<int64_t>((pieces + l.tx - 1) / l.tx, 1024 / blocks));
    auto *kernel = width < Vec<T>::n ? route_combine<T, false> : route_combine<T, true>;
    return launch("route_combine launch", kernel, spread(blocks, parts), dim3(kThreads), stream, static_cast<const T *>(rows), (long)ld_rows, weight,
                       row_of_slot, (long)tokens, k, (int)width, l.tx, static_cast<T *>(y), (long)ld_y);
}
// Few tokens: a token's slots, one trip to memory after another in one workgroup, are dealt to several (509 tokens of 1001 fp16, 8 slots: 12.8 us in one, 7.0 in eight).
int slots_a_workgroup(int64_t blocks, int k)
{
    const int64_t parts = std::max<int64_t>(1, std::min<int64_t>(k, 2048 / blocks));
    return (int)((k + parts - 1) / parts);
}
template <typename T>
int run_combine_grad(const void *dy, int64_t ld_dy, const void *rows, int64_t ld_rows, const float *weight, const int32_t *row_of_slot, const int32_t *held_at,
                     int64_t tokens, int k, int64_t width, void *drows, int64_t ld_drows, float *dweight, hipStream_t stream)
{
    const Lay l = lay_out((width + Vec<T>::n - 1) / Vec<T>::n, tokens, 1);
    const int64_t blocks = (tokens + l.ty - 1) / l.ty;
    const int share = slots_a_workgroup(blocks, k);
    auto *kernel = width < Vec<T>::n ? route_combine_grad<T, false> : route_combine_grad<T, true>;
    return launch("route_combine_grad launch", kernel, spread(blocks, (k + share - 1) / share), dim3(kThreads), stream, static_cast<const T *>(dy), (long)ld_dy,
                       static_cast<const T *>(rows), (long)ld_rows, weight, row_of_slot, held_at, (long)tokens, k, (int)width, l.tx, share, static_cast<T *>(drows),
                       (long)ld_drows, dweight);
}

}  // namespace

#define BY_DTYPE(dtype, call, ...)                                          \
    ((dtype) == OPEVO_F32 ? call<float>(__VA_ARGS__)                        \
     : (dtype) == OPEVO_BF16 ? call<__bf16>(__VA_ARGS__) : call<_Float16>(__VA_ARGS__))

extern "C" int opevo_route_workspace(int64_t tokens, int k, int experts, size_t *bytes)
{
    if (!bytes) return fail(OPEVO_E_ARG, "route_workspace: bytes is NULL");
    if (int rc = check_route("route_workspace", tokens, k, experts)) return rc;
    *bytes = workspace_of(tokens * k, experts);
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
    Route r = {};
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
    Route r = {};
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
