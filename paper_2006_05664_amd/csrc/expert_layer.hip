// A whole layer of experts for few tokens, in two launches:
//   h[s] = silu(x[t] Wg[e]^T) * (x[t] Wu[e]^T) for every slot s = (t, j) of expert e,   y[t] = sum_j weight[s] * (h[s] Wo[e]^T),
// weights in 8 bits with a scale a channel or in microscaled 4 bits (mx4.hpp), activations as they are.  What bounds it are the weights of the experts in use, each of which is read once; the
// products go through bf16 matrix instructions because those hold 8-bit integers and E2M1 values under their factors exactly.
//
// Activations of more bits go as a sum of bf16 numbers, each in a row of the product of its own: fp16 is the sum of two, fp32, and with it h, whatever the callers' type, of three: exactly, down to
// magnitudes of 2^-109, whose last bit is bf16's smallest number 2^-133, below which what they hold is cut off.  The product has 16 rows whatever they hold, so for the few rows of an expert
// the parts cost nothing, and the rows' sums are added at the end.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdint>

#include "launch.hpp"
#include "mx4.hpp"
#include "narrow.hpp"
#include "product.hpp"
#include "rows.hpp"

namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef int i32x2 __attribute__((ext_vector_type(2)));

constexpr int kMaxSlots = OPEVO_EXPERT_LAYER_MAX_SLOTS;
constexpr int kMaxExperts = OPEVO_ROUTE_MAX_EXPERTS;
constexpr int kStep = 128;              // values along K of four matrix instructions; lane (r, g) holds those from 32 g on of row r

// Some rows of one expert: `rows` of them from row `base` of h on, the `first`th and later ones of a group of tokens.
struct Unit { int expert, first, rows, base; };

// What the first launch leaves for the second, for every group of tokens (a group's slots are a stretch, and it has no more units than slots, which start where its slots do): its units and rows, and the
// place of each slot's row among the group's, or -1.
struct Plan {
    int units_of[kMaxSlots], rows_of[kMaxSlots], place[kMaxSlots];
    Unit units[kMaxSlots];
};

struct Layer {
    const void *x;
    long ld_x;
    const int *expert;
    const float *weight;
    int tokens, k, slots, experts, width, inner;
    const uint8_t *win, *wout;
    const void *sin, *sout;             // a float a channel, or a byte for 32 values
    long ld_in, ld_out, ld_sin, ld_sout;
    void *y;
    long ld_y;
    Plan *plan;
    int groups, group_tokens, group_unit;       // of the second launch: groups of tokens, how many tokens and how many rows of a unit
    __bf16 *h;                          // [held slots][parts][ld_h], zeros from `inner` on
    long ld_h;
};

// The high halves of two fp32 numbers: both as bf16, towards zero.
__device__ __forceinline__ int high_halves(float a, float b) { return (int)__builtin_amdgcn_perm(__float_as_uint(b), __float_as_uint(a), 0x07060302u); }
// What is left of a number without its first eight bits; of an infinity nothing.
__device__ __forceinline__ float rest(float v)
{
    const float high = __uint_as_float(__float_as_uint(v) & 0xffff0000u);
    return v == high ? 0.f : v - high;
}

// Where K ends: with an iteration, inside one, or before a row of weights has 16 bytes.
enum Ending { kEven, kRagged, kTiny };

// 16 bytes from byte `from` of a row that ends at byte `end`; what lies past it may be anything but has to be a number, as it meets activations of zero there.  A row of 16 bytes or more: its last 16,
// shifted, for the one piece that the row ends in (by as much for all lanes), and no branch, so that all pieces are on their way together.
template <Ending ENDING> __device__ __forceinline__ i32x4 load_end(const uint8_t *row, int from, int end)
{
    if (ENDING == kTiny) return load_chunk((const int8_t *)row, from, end);
    i32x4 v, w;
    __builtin_memcpy(&v, row + min(from, end - 16), 16);
    const int by = (16 - end % 16) % 16;
    w = by & 8 ? i32x4{v[2], v[3], 0, 0} : v;
    w = by & 4 ? i32x4{w[1], w[2], w[3], 0} : w;
    w = i32x4{(int)__builtin_amdgcn_alignbyte(w[1], w[0], by), (int)__builtin_amdgcn_alignbyte(w[2], w[1], by), (int)__builtin_amdgcn_alignbyte(w[3], w[2], by), (int)__builtin_amdgcn_alignbyte(0, w[3], by)};
    return from > end - 16 ? w : v;
}

// ------------------------------------------------------------------ weights
// Rows of weights, 16 of them to a tile: a lane has its row's pointer, loads 32 bytes of an iteration and makes of them the operands of SUB * 4 matrix instructions.
struct Weights8 {
    static constexpr int SUB = 1;
    struct Raw { i32x4 v[2]; };
    const uint8_t *row;
    int k;
    __device__ __forceinline__ void at(const uint8_t *w, long ld, const void *, long, long n, int k_) { row = w + n * ld; k = k_; }
    __device__ __forceinline__ void skip(int values) { row += values; }
    __device__ __forceinline__ void load(Raw &r, int k0, int g) const
    {
        __builtin_memcpy(&r.v[0], row + k0 + g * 32, 16);
        __builtin_memcpy(&r.v[1], row + k0 + g * 32 + 16, 16);
    }
    template <Ending ENDING> __device__ __forceinline__ void load_last(Raw &r, int k0, int g) const
    {
        r.v[0] = load_end<ENDING>(row, k0 + g * 32, k);
        r.v[1] = load_end<ENDING>(row, k0 + g * 32 + 16, k);
    }
    static __device__ __forceinline__ bf16x8 operand(const Raw &r, int, int j, int)
    {
        i32x4 out;
#pragma unroll
        for (int d = 0; d < 2; ++d) {
            const int w = r.v[j / 2][j % 2 * 2 + d];
            out[d * 2] = high_halves((float)(int8_t)w, (float)(int8_t)(w >> 8));
            out[d * 2 + 1] = high_halves((float)(int8_t)(w >> 16), (float)(w >> 24));
        }
        return __builtin_bit_cast(bf16x8, out);
    }
    static __device__ __forceinline__ float scale(const void *s, long channel) { return ((const float *)s)[channel]; }
};
struct Weights4 {
    static constexpr int SUB = 2;
    struct Raw { i32x4 v[2]; i32x2 f; };
    const uint8_t *row, *by;
    int k;                              // values
    __device__ __forceinline__ void at(const uint8_t *w, long ld, const void *s, long ld_s, long n, int k_) { row = w + n * ld; by = (const uint8_t *)s + n * ld_s; k = k_; }
    __device__ __forceinline__ void skip(int values)
    {
        row += values / 2;
        by += values / 32;
    }
    __device__ __forceinline__ void load(Raw &r, int k0, int g) const
    {
        __builtin_memcpy(&r.f, by + k0 / 32, 8);
        __builtin_memcpy(&r.v[0], row + k0 / 2 + g * 16, 16);
        __builtin_memcpy(&r.v[1], row + k0 / 2 + g * 16 + kStep / 2, 16);
    }
    template <Ending ENDING> __device__ __forceinline__ void load_last(Raw &r, int k0, int g) const
    {
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            // this lane's factor, where operand() looks for it; past the last one that one again
            r.f[u] = by[min(k0 / 32 + u * 4 + g, (k + 31) / 32 - 1)] << 8 * g;
            r.v[u] = load_end<ENDING>(row, k0 / 2 + g * 16 + u * (kStep / 2), (k + 1) / 2);
        }
    }
    static __device__ __forceinline__ bf16x8 operand(const Raw &r, int u, int j, int g)
    {
        const int w = r.v[u][j];
        const float by = mx4_factor((int)((unsigned)r.f[u] >> 8 * g & 255));
        const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, by, 0), b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, by, 1),
                     c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, by, 2), d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, by, 3);
        return bf16x8{a.x, a.y, b.x, b.y, c.x, c.y, d.x, d.y};
    }
    static __device__ __forceinline__ float scale(const void *, long) { return 1.f; }
};

// ------------------------------------------------------------------ activations
// How many bf16 numbers make one of a type, and what a row that holds the part `part` gives to the product.
template <typename T> struct Parts { static constexpr int n = 1, h = 3; };
template <> struct Parts<_Float16> { static constexpr int n = 2, h = 3; };
template <> struct Parts<float> { static constexpr int n = 3, h = 3; };

// Where value c of a row of h stands: the eight values that a lane takes of it at a time stand side by side with those that the lanes of the other three groups take at the same time, so that an
// access of the second launch is 64 contiguous bytes a row and not 16 of every 64.
__device__ __forceinline__ int place_in_h(int c) { return c / kStep * kStep + c % 32 / 8 * 32 + c % kStep / 32 * 8 + c % 8; }

template <typename T> __device__ __forceinline__ bf16x8 operand(const T (&v)[8], int part)
{
    if constexpr (Parts<T>::n == 1) {
        bf16x8 out;
        __builtin_memcpy(&out, v, 16);
        return out;
    } else {
        float f[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            f[i] = (float)v[i];
            const float second = rest(f[i]);
            if constexpr (Parts<T>::n == 2) f[i] = part == 0 ? f[i] : second;
            else f[i] = part == 0 ? f[i] : part == 1 ? second : rest(second);
        }
        const i32x4 out = {high_halves(f[0], f[1]), high_halves(f[2], f[3]), high_halves(f[4], f[5]), high_halves(f[6], f[7])};
        return __builtin_bit_cast(bf16x8, out);
    }
}

// A lane's row of activations.  A lane without one (`on` is false) loads nothing and multiplies what its registers hold: a column of the product is its row's alone.  (Loading some row instead
// costs as much as a row of its own: 32 tokens x 4 of 4096 x 1024, second launch, 49 us instead of 42.)
// `last` is a copy of an iteration that the row ends in, filled up with zeros, in the LDS.
template <typename T, int SUB> struct Activations {
    struct Raw { T v[SUB][4][8]; };
    const T *row, *last;
    int part, k;
    bool on;
    __device__ __forceinline__ void load(Raw &r, int k0, int g) const
    {
        if (!on) return;
#pragma unroll
        for (int u = 0; u < SUB; ++u)
#pragma unroll
            for (int j = 0; j < 4; ++j) __builtin_memcpy(r.v[u][j], row + k0 + u * kStep + g * 32 + j * 8, sizeof r.v[u][j]);
    }
    // the last iteration of a row that ends inside it, from the copy of it
    __device__ __forceinline__ void load_last(Raw &r, int g) const
    {
#pragma unroll
        for (int u = 0; u < SUB; ++u)
#pragma unroll
            for (int j = 0; j < 4; ++j) __builtin_memcpy(r.v[u][j], __builtin_assume_aligned(last + u * kStep + g * 32 + j * 8, 16), sizeof r.v[u][j]);
    }
};

// The iterations first, first + stride, ... along K, the last one of which may be ragged; the wave whose turn it is takes that one.  The weights of the next iteration come from memory meanwhile; the
// activations, of the same one, from the caches: they are asked for first, because loads are waited for in their order.
template <Ending ENDING, typename Q, typename T, int NI>
__device__ __forceinline__ void multiply(const Q (&w)[NI], const Activations<T, Q::SUB> &x, int first, int stride, int g, f32x4 (&acc)[NI])
{
    constexpr int LONG = Q::SUB * kStep;
    typedef typename Q::Raw W;
    typedef typename Activations<T, Q::SUB>::Raw X;
    const int whole = x.k / LONG;
    auto load = [&](W (&wr)[NI], int it) {
#pragma unroll
        for (int n = 0; n < NI; ++n) w[n].load(wr[n], it * LONG, g);
    };
    auto use = [&](const W (&wr)[NI], const X &xr) {
#pragma unroll
        for (int u = 0; u < Q::SUB; ++u)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const bf16x8 a = operand(xr.v[u][j], x.part);
#pragma unroll
                for (int n = 0; n < NI; ++n) acc[n] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(Q::operand(wr[n], u, j, g), a, acc[n], 0, 0, 0);
                __builtin_amdgcn_sched_barrier(0);      // operands are made as they are used: all at once they would take all registers
            }
        // The sums are due: else the compiler moves their products behind the next branch, with all their operands.
#pragma unroll
        for (int n = 0; n < NI; ++n) asm volatile("" : "+v"(acc[n]));
    };
    auto step = [&](const W (&wr)[NI], W (&next)[NI], int it) {
        X xr;
        x.load(xr, it * LONG, g);
        load(next, it + stride);
        use(wr, xr);
    };
    W wa[NI], wb[NI];
    // no load of weights in the loop stands behind a branch: a wait would be for those behind it too
    int it = first, left = first < whole ? (whole - first + stride - 1) / stride : 0;
    if constexpr (Parts<T>::n > 1 && Q::SUB == 2) {
        // one body where it is long, as its instructions have to come from memory too (4-bit weights, 1 token of 1967 x 768
        // in fp32 18 us, with three bodies 20; 102 x 2 of 8 experts, 246 x 2879 in fp16 53 and 61); past the last weights those again
        if (left > 0) load(wa, it);
        for (; left > 0; --left) {
            const int next = left > 1 ? it + stride : it;
            X xr;
            x.load(xr, it * LONG, g);
            load(wb, next);
            use(wa, xr);
#pragma unroll
            for (int n = 0; n < NI; ++n) wa[n] = wb[n];
            it = next;
        }
    } else if (left > 0) {
        load(wa, it);
        for (; left >= 3; left -= 2, it += 2 * stride) {
            step(wa, wb, it);
            step(wb, wa, it + stride);
        }
        if (left == 2) {
            step(wa, wb, it);
            it += stride;
#pragma unroll
            for (int n = 0; n < NI; ++n) wa[n] = wb[n];
        }
        X xr;
        x.load(xr, it * LONG, g);
        use(wa, xr);
    }
    if (ENDING != kEven && whole % stride == first) {
        X xr;
        x.load_last(xr, g);
#pragma unroll
        for (int n = 0; n < NI; ++n) w[n].template load_last<ENDING>(wa[n], whole * LONG, g);
        use(wa, xr);
    }
}

// ------------------------------------------------------------------ the first launch
// The slots' experts, held ones as they are and others as -1, and how many slots each expert has.
template <int NT> __device__ __forceinline__ void read_slots(const Layer &p, int *ids, int *counts)
{
    for (int e = threadIdx.x; e < p.experts; e += NT) counts[e] = 0;
    __syncthreads();
    for (int s = threadIdx.x; s < p.slots; s += NT) {
        const int e = p.expert[s];
        const bool held = (unsigned)e < (unsigned)p.experts;
        ids[s] = held ? e : -1;
        if (held) atomicAdd(&counts[e], 1);
    }
    __syncthreads();
}

// The sums of v over the lanes up to this one.
__device__ __forceinline__ int sum_upto(int v, int lane)
{
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const int up = __shfl_up(v, o);
        if (lane >= o) v += up;
    }
    return v;
}

// Exclusive sums of counts over the experts, by one wave, in place.
__device__ __forceinline__ void add_up(int *counts, int experts, int lane)
{
    int run = 0;
    for (int e0 = 0; e0 < experts; e0 += 64) {
        const int n = e0 + lane < experts ? counts[e0 + lane] : 0, upto = sum_upto(n, lane);
        if (e0 + lane < experts) counts[e0 + lane] = run + upto - n;
        run += __builtin_amdgcn_readlane(upto, 63);
    }
}

// The plan of one group of tokens, by one workgroup.  before: the slots of lower experts (rows of h are the held slots, sorted by expert); earlier, own: an expert's slots in front of the group
// and in it.
template <int NT> __device__ __forceinline__ void write_plan(const Layer &p, const int *ids, const int *before, int *earlier, int *own, int group, int lane)
{
    const int first = group * p.group_tokens * p.k, last = min(first + p.group_tokens * p.k, p.slots);
    __syncthreads();
    for (int e = threadIdx.x; e < p.experts; e += NT) earlier[e] = own[e] = 0;
    __syncthreads();
    for (int s = threadIdx.x; s < last; s += NT)
        if (ids[s] >= 0) atomicAdd(s < first ? &earlier[ids[s]] : &own[ids[s]], 1);
    __syncthreads();
    if (threadIdx.x < 64) {
        int units = 0, rows = 0;
        for (int e0 = 0; e0 < p.experts; e0 += 64) {
            const int e = e0 + lane, mine = e < p.experts ? own[e] : 0, n = (mine + p.group_unit - 1) / p.group_unit, upto = sum_upto(n, lane), rows_upto = sum_upto(mine, lane);
            const int at = rows + rows_upto - mine;
            for (int i = 0; i < n; ++i)
                p.plan->units[first + units + upto - n + i] = {e, at + i * p.group_unit, min(mine - i * p.group_unit, p.group_unit), before[e] + earlier[e] + i * p.group_unit};
            if (e < p.experts) own[e] = at;
            units += __builtin_amdgcn_readlane(upto, 63);
            rows += __builtin_amdgcn_readlane(rows_upto, 63);
        }
        if (lane == 0) {
            p.plan->units_of[group] = units;
            p.plan->rows_of[group] = rows;
        }
    }
    __syncthreads();
    for (int s = first + threadIdx.x; s < last; s += NT) {
        const int e = ids[s];
        int rank = 0;
        for (int o = first; o < s; ++o) rank += ids[o] == e;
        p.plan->place[s] = e < 0 ? -1 : own[e] + rank;
    }
}

// Every expert's rows make units of PER, the last one with fewer.  Unit number `index` of all; `first` counts the expert's rows.
template <int PER> __device__ __forceinline__ bool unit_at(const int *counts, int experts, int index, int lane, Unit *u)
{
    int seen = 0, base = 0;
    for (int e0 = 0; e0 < experts; e0 += 64) {
        const int n = e0 + lane < experts ? counts[e0 + lane] : 0, units = (n + PER - 1) / PER, upto = sum_upto(units, lane), rows = sum_upto(n, lane);
        const unsigned long long past = __ballot(seen + upto > index);
        if (past) {
            const int at = __ffsll(past) - 1, own = __builtin_amdgcn_readlane(n, at);
            u->expert = e0 + at;
            u->first = (index - seen - __builtin_amdgcn_readlane(upto - units, at)) * PER;
            u->rows = min(own - u->first, PER);
            u->base = base + __builtin_amdgcn_readlane(rows - n, at) + u->first;
            return true;
        }
        seen += __builtin_amdgcn_readlane(upto, 63);
        base += __builtin_amdgcn_readlane(rows, 63);
    }
    return false;
}

// h of a unit's rows for 16 * NP inner channels: gate and up, NP tiles of 16 rows of weights each, so that the operands of the activations serve 2 NP tiles.  The W waves deal the iterations
// along K among themselves.  NP is 2, or 1 where that would take more registers than there are: 4-bit weights whose rows end inside an iteration, activations in parts.
// Bound by the weights' bytes: 32 tokens x 4 of 64 experts, 4096 x 1024 in 4 bits, 144 MB in 34 - 41 us; for one token by a launch and a trip to memory: 2 of 8, 1024 x 4096 in 8 bits, 17 MB in 7.5.
template <typename T, typename Q, Ending ENDING> constexpr int kPairs = ENDING != kEven && Q::SUB == 2 && Parts<T>::n > 1 ? 1 : 2;
template <typename T, typename Q, int W, Ending ENDING>
__global__ __launch_bounds__(W * 64, 2)
void layer_in(Layer p)
{
    constexpr int NT = W * 64, NP = kPairs<T, Q, ENDING>, NI = 2 * NP, LONG = Q::SUB * kStep, PX = Parts<T>::n, PH = Parts<T>::h, PER = 16 / PX;
    __shared__ int ids[kMaxSlots], counts[kMaxExperts], token[PER];
    __shared__ f32x4 sums[W][NI][64];
    __shared__ __attribute__((aligned(16))) T last[ENDING == kEven ? 1 : PER][LONG];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), g = lane >> 4, r = lane & 15, c0 = blockIdx.x * (NP * 16);
    read_slots<NT>(p, ids, counts);
    if (blockIdx.y == gridDim.y - 1) {
        if (threadIdx.x < 64) add_up(counts, p.experts, lane);
        int *const more = (int *)sums;
        static_assert(sizeof sums >= 2 * kMaxExperts * sizeof(int), "");
        for (int group = blockIdx.x; group < p.groups; group += gridDim.x) write_plan<NT>(p, ids, counts, more, more + kMaxExperts, group, lane);
        return;
    }
    Unit unit;
    if (!unit_at<PER>(counts, p.experts, blockIdx.y, lane, &unit)) return;         // alike for the workgroup
    if (wave == 0)
        for (int s0 = 0, seen = -unit.first; s0 < p.slots && seen < unit.rows; s0 += 64) {
            const bool mine = s0 + lane < p.slots && ids[s0 + lane] == unit.expert;
            const unsigned long long same = __ballot(mine);
            const int at = seen + __popcll(same & ((1ull << lane) - 1ull));
            if (mine && at >= 0 && at < unit.rows) token[at] = (s0 + lane) / p.k;
            seen += __popcll(same);
        }
    __syncthreads();
    const long first = (long)unit.expert * 2 * p.inner;
    Q w[NI];
#pragma unroll
    for (int n = 0; n < NI; ++n) w[n].at(p.win, p.ld_in, p.sin, p.ld_sin, first + (n < NP ? 0 : p.inner) + min(c0 + n % NP * 16 + r, p.inner - 1), p.width);
    Activations<T, Q::SUB> x;
    x.on = r < unit.rows * PX;
    x.row = (const T *)p.x + token[min(r / PX, unit.rows - 1)] * p.ld_x;
    x.part = r % PX;
    x.k = p.width;
    if (ENDING != kEven) {
        const int whole = p.width / LONG * LONG;
        for (int i = threadIdx.x; i < unit.rows * LONG; i += NT) {
            const int c = whole + i % LONG;
            last[i / LONG][i % LONG] = c < p.width ? ((const T *)p.x)[token[i / LONG] * p.ld_x + c] : (T)0.f;
        }
        __syncthreads();
        x.last = last[min(r / PX, unit.rows - 1)];
    }
    f32x4 acc[NI] = {};
    multiply<ENDING, Q, T, NI>(w, x, wave, W, g, acc);
#pragma unroll
    for (int n = 0; n < NI; ++n) sums[wave][n][lane] = acc[n];
    __syncthreads();
    // an output a thread: one inner channel of one row
    for (int o = threadIdx.x; o < unit.rows * NP * 16; o += NT) {
        const int c = o % (NP * 16), at = o / (NP * 16);
        if (c0 + c >= p.ld_h) continue;
        __bf16 *to = p.h + (long)(unit.base + at) * PH * p.ld_h + place_in_h(c0 + c);
        if (c0 + c >= p.inner) {
#pragma unroll
            for (int part = 0; part < PH; ++part) to[part * p.ld_h] = (__bf16)0.f;
            continue;
        }
        float v[2] = {0.f, 0.f};
#pragma unroll
        for (int side = 0; side < 2; ++side)
#pragma unroll
            for (int part = PX - 1; part >= 0; --part)
                for (int o = 0; o < W; ++o) v[side] += ((const float *)&sums[o][side * NP + c / 16][c % 16 / 4 * 16 + at * PX + part])[c % 4];
        const float gate = v[0] * Q::scale(p.sin, first + c0 + c), up = v[1] * Q::scale(p.sin, first + p.inner + c0 + c);
        const float h = gate / (1.f + expf(-gate)) * up, second = rest(h);
        static_assert(PH == 3, "");
        to[0] = __builtin_bit_cast(__bf16, (unsigned short)(__float_as_uint(h) >> 16));
        to[p.ld_h] = __builtin_bit_cast(__bf16, (unsigned short)(__float_as_uint(second) >> 16));
        to[2 * p.ld_h] = __builtin_bit_cast(__bf16, (unsigned short)(__float_as_uint(rest(second)) >> 16));
    }
}

// ------------------------------------------------------------------ the second launch
// y of NC tiles of COLS = 16 / S columns for a group of tokens: a task is a unit of rows of an expert and a share of K, the W waves deal the tasks among themselves, what they find for each row
// meets in LDS, and the rows of a token are added up there in the order of its slots.  A wave goes through its tasks' iterations as one sequence, the next two on their way from memory whichever task
// they belong to: an iteration is a few microseconds' worth of latency and a fraction of one of work.
// S > 1, for few columns: K falls into S parts, and the 16 rows of weights of a product are COLS columns in each of the parts, the 16 rows of h COLS rows in each of
// them.  Of the product the S blocks of a part with itself are used; a wave reads as much as ever, and there are S times as many workgroups.
// Of the same layers: 82 MB in 31 - 32 us, 9 MB in 7.8 - 8.2.
constexpr int kShares = 1024;           // rows of 16 sums, or of the 32 of two tiles, in the LDS
constexpr unsigned kNowhere = 0xf0000000u;      // behind the end of h, which has 3 * 2^30 bytes at most, with whatever is added to it

template <typename T, typename Q, int W, int S, int NC, Ending ENDING>
__global__ __launch_bounds__(W * 64)
void layer_out(Layer p)
{
    constexpr int NT = W * 64, COLS = 16 / S, WIDE = NC * COLS, PH = Parts<T>::h, PER = COLS / PH, LONG = Q::SUB * kStep;
    static_assert(PER >= 1 && (S == 1 || (ENDING == kEven && NC == 1)), "");
    __shared__ int place[kMaxSlots];
    __shared__ float by[kMaxSlots];
    __shared__ Unit units[kMaxSlots];
    __shared__ __attribute__((aligned(16))) float z[kShares * S][WIDE];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), g = lane >> 4, r = lane & 15, part = r / COLS, c = r % COLS, n0 = blockIdx.x * WIDE;
    const int t0 = blockIdx.y * p.group_tokens, tokens = min(p.group_tokens, p.tokens - t0), first = t0 * p.k;
    const int all = __builtin_amdgcn_readfirstlane(p.plan->units_of[blockIdx.y]), here = __builtin_amdgcn_readfirstlane(p.plan->rows_of[blockIdx.y]);
    for (int s = threadIdx.x; s < tokens * p.k; s += NT) {
        place[s] = p.plan->place[first + s];
        by[s] = p.weight ? p.weight[first + s] : 1.f;
        units[s] = p.plan->units[first + s];
    }
    __syncthreads();
    const int length = p.inner / S, whole = length / LONG, count = (length + LONG - 1) / LONG;
    // shares of K: as many as make the waves' iterations fewest, one lost to each task
    int shares = 1, least = INT32_MAX;
    for (int s = 1; s <= W && s <= count && s * here <= kShares; s *= 2) {
        const int cost = (all * s + W - 1) / W * ((count + s - 1) / s + 1);
        if (cost < least) { least = cost; shares = s; }
    }
    const int shift = __builtin_ctz(shares), tasks = all * shares;

    // The wave's tasks, every W-th, all of the same share of K, and their iterations: as they are loaded and as they are used.
    const int share = wave & (shares - 1), own = (tasks - wave + W - 1) / W;
    int load_task = wave, load_it = share, use_task = wave, use_it = share;
    Q w[NC];
    // rows of h as a buffer, whose bounds answer for lanes without a row: zeros, and no access
    const __amdgpu_buffer_rsrc_t h = __builtin_amdgcn_make_buffer_rsrc(p.h, 0, (int)(unsigned)((long)p.slots * PH * p.ld_h * 2), 0x00027000);
    unsigned row_at = 0;
    auto aim = [&](int task) {
        const Unit unit = units[task >> shift];
        const int e = __builtin_amdgcn_readfirstlane(unit.expert), base = __builtin_amdgcn_readfirstlane(unit.base), rows = __builtin_amdgcn_readfirstlane(unit.rows);
#pragma unroll
        for (int n = 0; n < NC; ++n) {
            w[n].at(p.wout, p.ld_out, p.sout, p.ld_sout, (long)e * p.width + min(n0 + n * COLS + c, p.width - 1), p.inner);
            if (S > 1) w[n].skip(part * length);
        }
        row_at = c < rows * PH ? (((base + c / PH) * PH + c % PH) * (unsigned)p.ld_h + part * length + g * 8) * 2 : kNowhere;
    };
    struct Buffer { typename Q::Raw w[NC]; i32x4 x[Q::SUB][4]; } b0, b1, b2;
    auto load = [&](Buffer &b) {
#pragma unroll
        for (int u = 0; u < Q::SUB; ++u)
#pragma unroll
            for (int j = 0; j < 4; ++j) b.x[u][j] = __builtin_amdgcn_raw_buffer_load_b128(h, row_at + (load_it * LONG + u * kStep + j * 32) * 2, 0, 0);
#pragma unroll
        for (int n = 0; n < NC; ++n) {
            if (ENDING == kEven || load_it < whole) w[n].load(b.w[n], load_it * LONG, g);
            else w[n].template load_last<ENDING>(b.w[n], load_it * LONG, g);
        }
        load_it += shares;
        if (load_it >= count && load_task + W < tasks) {
            load_it = share;
            load_task += W;
            aim(load_task);
        }
    };
    f32x4 acc[NC] = {};
    auto use = [&](const Buffer &b) {
#pragma unroll
        for (int u = 0; u < Q::SUB; ++u)
#pragma unroll
            for (int j = 0; j < 4; ++j)
#pragma unroll
                for (int n = 0; n < NC; ++n) acc[n] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(Q::operand(b.w[n], u, j, g), __builtin_bit_cast(bf16x8, b.x[u][j]), acc[n], 0, 0, 0);
#pragma unroll
        for (int n = 0; n < NC; ++n) asm volatile("" : "+v"(acc[n]));           // due here, not behind the next branch
        use_it += shares;
        if (use_it < count) return;
        const Unit unit = units[use_task >> shift];
#pragma unroll
        for (int n = 0; n < NC; ++n) {
            f32x4 v;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                float sum = acc[n][i];
#pragma unroll
                for (int o = 1; o < PH; ++o) sum += __shfl_down(acc[n][i], o);
                v[i] = sum;
            }
            // lane (r, g) has the sums of rows 4 g .. 4 g + 3 of the weights with row r of h
            if (g * 4 / COLS == part && c < unit.rows * PH && c % PH == 0)
                *(f32x4 *)&z[(share * S + part) * here + unit.first + c / PH][n * COLS + g * 4 % COLS] = v;
            acc[n] = f32x4{0.f, 0.f, 0.f, 0.f};
        }
        use_it = share;
        use_task += W;
    };
    // Two iterations are on their way while one is used.  In the loop no load stands behind a branch: waits there would be for all loads, as if those behind it had not been.
    int left = own > 0 ? own * ((count - share + shares - 1) / shares) : 0;
    if (left > 0) aim(wave);
    if (left >= 2) {
        load(b0);
        load(b1);
        for (; left >= 5; left -= 3) {
            load(b2);
            use(b0);
            load(b0);
            use(b1);
            load(b1);
            use(b2);
        }
        if (left >= 3) load(b2);
        use(b0);
        if (left >= 4) load(b0);
        use(b1);
        if (left >= 3) use(b2);
        if (left >= 4) use(b0);
    } else if (left == 1) {
        load(b0);
        use(b0);
    }
    __syncthreads();
    for (int o = threadIdx.x; o < tokens * WIDE; o += NT) {
        const int t = o / WIDE, col = o % WIDE;
        if (n0 + col >= p.width) continue;
        float y = 0.f;
        for (int j0 = 0; j0 < p.k; j0 += 4) {           // four scales on their way
            float scale[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int s = t * p.k + min(j0 + j, p.k - 1);
                scale[j] = place[s] < 0 ? 0.f : Q::scale(p.sout, (long)p.expert[first + s] * p.width + n0 + col);
            }
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int s = t * p.k + j0 + j, row = j0 + j < p.k ? place[s] : -1;
                if (row < 0) continue;
                float sum = 0.f;
                for (int u = 0; u < shares * S; ++u) sum += z[u * here + row][col];
                y = fmaf(by[s], sum * scale[j], y);
            }
        }
        ((T *)p.y)[(t0 + t) * p.ld_y + n0 + col] = narrow<T>(y);
    }
}

// ------------------------------------------------------------------ host side
using opevo::launch;

int check_layer(const char *who, int64_t tokens, int k, int experts, int dtype, int64_t width, int64_t inner)
{
    if (!known(dtype)) return fail(OPEVO_E_ARG, "%s: unknown element type %d", who, dtype);
    if (tokens < 0 || k < 1 || k > OPEVO_ROUTE_MAX_SLOTS || tokens > kMaxSlots / k)
        return fail(OPEVO_E_ARG, "%s: tokens %lld with %d slots each (1 to %d, %d in all)", who, (long long)tokens, k, OPEVO_ROUTE_MAX_SLOTS, kMaxSlots);
    if (experts < 1 || experts > OPEVO_ROUTE_MAX_EXPERTS) return fail(OPEVO_E_ARG, "%s: %d experts (1 to %d)", who, experts, OPEVO_ROUTE_MAX_EXPERTS);
    constexpr int64_t most = 1 << 20;
    if (width < 1 || width > most || inner < 1 || inner > most)
        return fail(OPEVO_E_ARG, "%s: %lld channels and %lld inner ones (1 to 2^20)", who, (long long)width, (long long)inner);
    return OPEVO_OK;
}

int64_t row_of_h(int64_t inner) { return (inner + 2 * kStep - 1) / (2 * kStep) * (2 * kStep); }
size_t layer_workspace(int64_t slots, int64_t inner) { return sizeof(Plan) + (size_t)slots * Parts<float>::h * row_of_h(inner) * sizeof(__bf16); }

template <typename T, typename Q>
int run_layer(Layer p, hipStream_t stream)
{
    constexpr int LONG = Q::SUB * kStep, PER = 16 / Parts<T>::n;
    const auto ending = [](int k) { return k % LONG == 0 ? kEven : k < (Q::SUB == 1 ? 16 : 31) ? kTiny : kRagged; };
    const Ending in = ending(p.width), of = ending(p.inner);
    // The second launch: a workgroup to 16 columns for each compute unit, or parts of K as long as that leaves units without one and the slots are few: parts leave room for fewer rows of an expert in a
    // product, whose weights are then read once more for the others (us, whole layers, S = 1 / 2 / 4: 1024 columns of 4096 inner ones, 1 token x 8 of 64 experts in 8 bits 48 / 39 / 34, 16 x 2 of 8 in
    // 4 bits 36 / 37 / 51, 100 x 2 of 8 in 8 bits 100 / 154 / 265; 256 of 1024, 4 x 4 of 32 in fp32 17 / 15 / 15, 32 x 4 of 64 in 4 bits 25 / 26 / 29; 2048 of 1024, 1 x 8 of 64 22 / 20 / 21, 100 x 2 of
    // 8 52 / 85 / 139) ...
    const int tiles = (p.width + 15) / 16, work = p.slots * tiles;
    int parts = tiles <= 80 ? (work < 1024 ? 4 : work <= 4096 ? 2 : 1) : tiles <= 160 && work < 1024 ? 2 : 1;
    while (parts > 1 && (p.inner % (parts * LONG) != 0 || 16 / parts < Parts<T>::h)) parts /= 2;
    // for many slots 32 columns a workgroup, which halve what it reads of h for its weights (us, whole layers, 32 columns / 16: 32 tokens x 4 of 64 experts, 4096 x 1024 in 4 bits 105 / 108; 63 x 5 of 72,
    // 2983 x 640 in fp16 135 / 156; 64 x 8 of 64, 4096 x 1024 in 8 bits 235 / 291; 5 x 6 of 9, 2048 x 1868 44 / 36)
    const bool wide = parts == 1 && p.slots >= 80 && p.width >= 1024;
    auto *out = wide ? (of == kTiny ? layer_out<T, Q, 8, 1, 2, kTiny> : of == kRagged ? layer_out<T, Q, 8, 1, 2, kRagged> : layer_out<T, Q, 8, 1, 2, kEven>)
                : of == kTiny ? layer_out<T, Q, 8, 1, 1, kTiny> : of == kRagged ? layer_out<T, Q, 8, 1, 1, kRagged>
                : parts == 4 ? layer_out<T, Q, 8, 4, 1, kEven> : parts == 2 ? layer_out<T, Q, 8, 2, 1, kEven> : layer_out<T, Q, 8, 1, 1, kEven>;
    // ... and where that is not enough the tokens in groups, each of which reads its experts' weights again, mostly from the caches (us, groups / one: 4-bit weights, 102 tokens x 2 of 8 experts, 246
    // columns of 2879 inner ones, fp16 57 / 169; 126 x 1 of 15, 469 of 1280, fp32 50 / 82; 8 bits, 32 x 1 of 62, 64 of 525 11 / 27)
    const int cols = wide ? 32 : 16 / parts, across = (p.width + cols - 1) / cols;
    p.groups = std::min(p.tokens, std::max(1, 256 / across));
    p.group_tokens = (p.tokens + p.groups - 1) / p.groups;
    p.groups = (p.tokens + p.group_tokens - 1) / p.group_tokens;
    p.group_unit = 16 / parts / Parts<T>::h;

    const int units = std::min(p.slots, std::min(p.slots, p.experts) + p.slots / PER);      // of the first launch; there can be no more
    const int channels = 16 * (in == kEven ? kPairs<T, Q, kEven> : kPairs<T, Q, kRagged>);
    auto *first = in == kEven ? layer_in<T, Q, 4, kEven> : in == kRagged ? layer_in<T, Q, 4, kRagged> : layer_in<T, Q, 4, kTiny>;
    if (int rc = launch("layer_in launch", first, dim3((unsigned)(p.ld_h / channels), units + 1), dim3(256), stream, p)) return rc;
    return launch("layer_out launch", out, dim3(across, p.groups), dim3(512), stream, p);
}
template <typename T> int run_layer8(const Layer &p, hipStream_t stream) { return run_layer<T, Weights8>(p, stream); }
template <typename T> int run_layer4(const Layer &p, hipStream_t stream) { return run_layer<T, Weights4>(p, stream); }

// The checks that both kinds of weights share, and where things stand in the workspace.
int plan_layer(const char *who, Layer *p, int dtype, int64_t tokens, int k, int experts, int64_t width, int64_t inner, void *workspace, size_t bytes)
{
    const size_t size = size_of(dtype);
    if (int rc = check_rows(who, "x", p->x, p->ld_x, width, size)) return rc;
    if (int rc = check_rows(who, "y", p->y, p->ld_y, width, size)) return rc;
    if (int rc = check_words(who, "expert", p->expert)) return rc;
    if (!aligned(p->weight, 4)) return fail(OPEVO_E_ARG, "%s: weight is not aligned to 4 bytes", who);
    const size_t need = layer_workspace(tokens * k, inner);
    if (!workspace || !aligned(workspace, 16) || bytes < need)
        return fail(OPEVO_E_ARG, "%s: the workspace holds %zu bytes of the %zu it takes, or is not aligned to 16 bytes", who, workspace ? bytes : 0, need);
    p->tokens = (int)tokens; p->k = k; p->slots = (int)tokens * k; p->experts = experts; p->width = (int)width; p->inner = (int)inner;
    p->plan = static_cast<Plan *>(workspace);
    p->h = reinterpret_cast<__bf16 *>(p->plan + 1);
    p->ld_h = row_of_h(inner);
    return OPEVO_OK;
}

}  // namespace

extern "C" int opevo_expert_layer_workspace(int64_t tokens, int k, int dtype, int64_t inner, size_t *bytes)
{
    const char *who = "expert_layer_workspace";
    if (!bytes) return fail(OPEVO_E_ARG, "%s: bytes is NULL", who);
    if (int rc = check_layer(who, tokens, k, 1, dtype, 1, inner)) return rc;
    *bytes = tokens == 0 ? 0 : layer_workspace(tokens * k, inner);
    return OPEVO_OK;
}

extern "C" int opevo_expert_layer_i8(const void *x, int64_t ld_x, int dtype, const int32_t *expert, const float *weight, int64_t tokens, int k, int experts, int64_t width,
                                     int64_t inner, const int8_t *w_in, int64_t ld_in, const float *scale_in, const int8_t *w_out, int64_t ld_out, const float *scale_out,
                                     void *y, int64_t ld_y, void *workspace, size_t workspace_bytes, void *stream)
{
    const char *who = "expert_layer_i8";
    if (int rc = check_layer(who, tokens, k, experts, dtype, width, inner)) return rc;
    if (tokens == 0) return OPEVO_OK;
    Layer p = {};
    p.x = x; p.ld_x = (long)ld_x; p.expert = expert; p.weight = weight; p.y = y; p.ld_y = (long)ld_y;
    p.win = reinterpret_cast<const uint8_t *>(w_in); p.ld_in = (long)ld_in; p.sin = scale_in;
    p.wout = reinterpret_cast<const uint8_t *>(w_out); p.ld_out = (long)ld_out; p.sout = scale_out;
    if (int rc = check_rows(who, "w_in", w_in, ld_in, width, 1)) return rc;
    if (int rc = check_words(who, "scale_in", scale_in)) return rc;
    if (int rc = check_rows(who, "w_out", w_out, ld_out, inner, 1)) return rc;
    if (int rc = check_words(who, "scale_out", scale_out)) return rc;
    if (int rc = plan_layer(who, &p, dtype, tokens, k, experts, width, inner, workspace, workspace_bytes)) return rc;
    return BY_DTYPE(dtype, run_layer8, p, static_cast<hipStream_t>(stream));
}

extern "C" int opevo_expert_layer_mx4(const void *x, int64_t ld_x, int dtype, const int32_t *expert, const float *weight, int64_t tokens, int k, int experts, int64_t width,
                                      int64_t inner, const uint8_t *w_in, int64_t ld_in, const uint8_t *scale_in, int64_t ld_scale_in, const uint8_t *w_out, int64_t ld_out,
                                      const uint8_t *scale_out, int64_t ld_scale_out, void *y, int64_t ld_y, void *workspace, size_t workspace_bytes, void *stream)
{
    const char *who = "expert_layer_mx4";
    if (int rc = check_layer(who, tokens, k, experts, dtype, width, inner)) return rc;
    if (tokens == 0) return OPEVO_OK;
    Layer p = {};
    p.x = x; p.ld_x = (long)ld_x; p.expert = expert; p.weight = weight; p.y = y; p.ld_y = (long)ld_y;
    p.win = w_in; p.ld_in = (long)ld_in; p.sin = scale_in; p.ld_sin = (long)ld_scale_in;
    p.wout = w_out; p.ld_out = (long)ld_out; p.sout = scale_out; p.ld_sout = (long)ld_scale_out;
    if (int rc = check_rows(who, "w_in", w_in, ld_in, (width + 1) / 2, 1)) return rc;
    if (int rc = check_rows(who, "scale_in", scale_in, ld_scale_in, (width + 31) / 32, 1)) return rc;
    if (int rc = check_rows(who, "w_out", w_out, ld_out, (inner + 1) / 2, 1)) return rc;
    if (int rc = check_rows(who, "scale_out", scale_out, ld_scale_out, (inner + 31) / 32, 1)) return rc;
    if (int rc = plan_layer(who, &p, dtype, tokens, k, experts, width, inner, workspace, workspace_bytes)) return rc;
    return BY_DTYPE(dtype, run_layer4, p, static_cast<hipStream_t>(stream));
}
