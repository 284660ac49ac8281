// Products of 8-bit integers with a scale for each row of either operand:
//   C[m, n] = (sum_k A[m, k] B[n, k]) * (sa[m] * sb[n]),
// the sum in 32-bit integers, exactly (K < 2^17, so that 128 * 128 * K fits), one rounding of it to fp32, one for each product, and one to
// the output type.  B holds an output channel a row, as the weights of a layer are stored, so both operands are read along K.  The grouped form gives each
// range of rows offsets[e] .. offsets[e + 1] a B of its own; the offsets are known on the device only.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdint>

#include "launch.hpp"
#include "narrow.hpp"
#include "wave.hpp"

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

// A grid's second extent ends at 65535: tiles of rows go on in the third.
constexpr int kGridY = 65535;
__device__ __forceinline__ long row_tile() { return (long)blockIdx.z * kGridY + blockIdx.y; }

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

// Writes a wave's MI x NI atoms, rows r.first + m0 .. and columns col0 .. of C.  Atom (i, j): lane l holds columns 4 * (l / 16) .. + 3 of row l % 16 (the MFMA takes B's
// rows as its first operand).  Stored like that, an instruction would touch 16 rows, 32 bytes of each, and the scales would be loaded under a mask for every atom
// (8192 x 4096 x 1024: 77 us, 27 of them for each tile's epilogue); the 16 rows of an atom row go through a piece of LDS of the wave's own instead and leave as whole
// lines, 16 bytes a lane.
template <typename T, int NI> constexpr int kPatch = 16 * NI * 16 * (int)sizeof(T);   // bytes of LDS a wave takes
template <typename T, int MI, int NI>
__device__ __forceinline__ void store_tile(const Product &p, const Rows &r, int m0, int col0, const i32x4 (&acc)[MI][NI], int8_t *patch, int lane)
{
    constexpr int PITCH = NI * 16 * (int)sizeof(T), CPR = NI * (int)sizeof(T), V = 16 / (int)sizeof(T);   // bytes, 16-byte chunks of a row, elements of a chunk
    static_assert((CPR & (CPR - 1)) == 0, "chunks are permuted by an exclusive or");
    const int cols = p.n - col0;
    const float *sbp = p.sb + (long)r.expert * p.n + col0;
    float sb[NI][4], sa[MI];
#pragma unroll
    for (int j = 0; j < NI; ++j) {
        const int c = j * 16 + (lane >> 4) * 4;
        if (!r.zero && c + 4 <= cols) __builtin_memcpy(sb[j], sbp + c, 16);
        else
#pragma unroll
            for (int e = 0; e < 4; ++e) sb[j][e] = !r.zero && c + e < cols ? sbp[c + e] : 0.f;
    }
#pragma unroll
    for (int i = 0; i < MI; ++i) {
        const long m = r.first + m0 + i * 16 + (lane & 15);
        sa[i] = !r.zero && m < r.last ? p.sa[m] : 0.f;
    }
#pragma unroll
    for (int i = 0; i < MI; ++i) {
#pragma unroll
        for (int j = 0; j < NI; ++j) {
            T v[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] = narrow<T>((float)acc[i][j][e] * (sa[i] * sb[j][e]));
            constexpr int OF = 16 / (4 * (int)sizeof(T));       // such pieces of a chunk
            const int piece = j * 4 + (lane >> 4), chunk = (piece / OF) ^ (lane & 15) % CPR;     // a row's chunks are permuted, so that 16 rows fall on different banks
            __builtin_memcpy(__builtin_assume_aligned(patch + (lane & 15) * PITCH + chunk * 16 + piece % OF * (16 / OF), 4 * sizeof(T)), v, sizeof v);
        }
        exchange();
        const long row0 = r.first + m0 + i * 16;
#pragma unroll
        for (int u = 0; u < (16 * CPR + 63) / 64; ++u) {
            const int at = u * 64 + lane, row = at / CPR, c = at % CPR * V;
            if ((16 * CPR) % 64 != 0 && row >= 16) continue;
            if (row0 + row >= r.last || c >= cols) continue;
            T *dst = (T *)p.c + (row0 + row) * p.ldc + col0 + c;
            const int8_t *from = patch + row * PITCH + (at % CPR ^ row % CPR) * 16;
            if (c + V <= cols) __builtin_memcpy(dst, __builtin_assume_aligned(from, 16), 16);
            else
#pragma unroll 1
                for (int e = 0; e < cols - c; ++e) dst[e] = ((const T *)from)[e];
        }
        exchange();
    }
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

// ------------------------------------------------------------------ few rows
// For few rows the weights are all there is to read, each once, and the time is that of one trip to memory.  No LDS and no barrier stands between: every wave loads
// its fragments from global memory into registers, 256 values along K a step (four MFMA steps), the next step's while it multiplies.  The W waves of a
// workgroup share a tile of MI x NI atoms and deal the steps among themselves; their sums meet in LDS.  Loads take any alignment.  One row of 4096 x 1024 weights 3.5 us (a launch alone
// takes 2.3), of 8192 x 8192 15 us = 4.4 TB/s; 16 rows of it 18.  Wider tiles (1 x 2, 2 x 1 and 2 x 2 atoms) and 8 or 16 waves measured the same or slower.
template <int MI, int NI, int W>
__global__ __launch_bounds__(W * 64)
void product_thin(Product p)
{
    __shared__ i32x4 sums[W][MI * NI][64];
    Rows r;
    if (!find_rows(p, MI * 16, row_tile(), &r)) return;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), n0 = blockIdx.x * NI * 16;
    i32x4 acc[MI][NI] = {};
    if (!r.zero) {
        const int8_t *row[MI + NI];
#pragma unroll
        for (int i = 0; i < MI; ++i) {
            const long m = r.first + i * 16 + (lane & 15);
            row[i] = p.a + (m < r.last ? m : r.last - 1) * p.lda;
        }
#pragma unroll
        for (int j = 0; j < NI; ++j) {
            const int n = n0 + j * 16 + (lane & 15);
            row[MI + j] = p.b + ((long)r.expert * p.n + (n < p.n ? n : p.n - 1)) * p.ldb;
        }
        const int kl = (lane >> 4) * 16, steps = (p.k + 255) / 256;
        i32x4 v[MI + NI][4], w[MI + NI][4];
        auto load = [&](i32x4 (&to)[MI + NI][4], int step) {
            const int k0 = step * 256 + kl;
            if (step * 256 + 256 <= p.k) {
#pragma unroll
                for (int i = 0; i < MI + NI; ++i)
#pragma unroll
                    for (int u = 0; u < 4; ++u) __builtin_memcpy(&to[i][u], row[i] + k0 + u * 64, 16);
            } else {
#pragma unroll
                for (int i = 0; i < MI + NI; ++i)
#pragma unroll
                    for (int u = 0; u < 4; ++u) to[i][u] = load_chunk(row[i], k0 + u * 64, p.k);
            }
        };
        auto multiply = [&](const i32x4 (&of)[MI + NI][4]) {
#pragma unroll
            for (int u = 0; u < 4; ++u)
#pragma unroll
                for (int i = 0; i < MI; ++i)
#pragma unroll
                    for (int j = 0; j < NI; ++j) acc[i][j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(of[MI + j][u], of[i][u], acc[i][j], 0, 0, 0);
        };
        int s = wave;
        if (s < steps) load(v, s);
        for (; s < steps; s += 2 * W) {
            if (s + W < steps) load(w, s + W);
            multiply(v);
            if (s + W >= steps) break;
            if (s + 2 * W < steps) load(v, s + 2 * W);
            multiply(w);
        }
    }
#pragma unroll
    for (int i = 0; i < MI; ++i)
#pragma unroll
        for (int j = 0; j < NI; ++j) sums[wave][i * NI + j][lane] = acc[i][j];
    __syncthreads();
    for (int at = wave; at < MI * NI; at += W) {
        i32x4 sum = sums[0][at][lane];
#pragma unroll
        for (int o = 1; o < W; ++o) sum += sums[o][at][lane];
        const long m = r.first + at / NI * 16 + (lane & 15);
        const int col = n0 + at % NI * 16 + (lane >> 4) * 4;
        if (m >= r.last) continue;
        const float *sb = p.sb + (long)r.expert * p.n + col;
        const float sa = r.zero ? 0.f : p.sa[m];
        float c[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) c[e] = !r.zero && col + e < p.n ? (float)sum[e] * (sa * sb[e]) : 0.f;
        if (p.out == OPEVO_F32) store4((float *)p.c + m * p.ldc, col, p.n, c);
        else if (p.out == OPEVO_BF16) store4((__bf16 *)p.c + m * p.ldc, col, p.n, c);
        else store4((_Float16 *)p.c + m * p.ldc, col, p.n, c);
    }
}

// ------------------------------------------------------------------ tiles
// Workgroup tile BM x BN, slabs of 128 values, WM x WN waves of MI x NI atoms of 16 x 16 x 64, KG groups of such waves that take every KG-th slab and add up
// their sums in LDS at the end (for grids that leave a compute unit one workgroup, whose slabs are a chain of latencies).  The 16-byte chunk c of a row sits at chunk
// position c ^ (row / 2 % 8) of its row of the slab: the 16 lanes of a turn of a fragment read then fall on 16 different groups of banks.
// Rows past the end repeat the last one (their results are not stored); chunks past K are zeros.
// DIRECT: every wave issues wave-wide loads of 16 bytes a lane whose destination is LDS, eight rows of a slab an instruction, the chunk each lane loads chosen by the
// permutation; a ring of STAGES slabs keeps STAGES - 1 in flight.  For operands whose pointers, row lengths and K are multiples of 16.
// Otherwise the slabs pass through registers, from where they start on any address: two stages in LDS, the slab after them on its way.
// 8192^3: 256 x 256 tiles 416 - 433 us (2540 - 2640 TOP/s), matrix pipes 64 % busy; 386 with zero operands (power), 333 when all rows are the same (memory).  More stages of
// shorter slabs 455, two workgroups of 256 x 128 a unit 525, 16 waves 732, 4 waves of 128 x 128 597, a workgroup that goes from tile to tile 426; through registers in
// 128 x 256 tiles 552, and 4095^3, whose rows start anywhere, 114 (4096^3 60): 16 bytes from any address are 6.6 times as many
// accesses of the L1 as 4096^3 makes, and the units that take the addresses apart are busy for 69 % of the time (40 %).  1000 x 1000 x 1008 in 64 x 64 tiles 5.7, 1000 x 1000 x 1001 7.7.
template <bool DIRECT_, int BM_, int BN_, int WM_, int WN_, int STAGES_, int KG_ = 1>
struct Shape {
    static constexpr bool DIRECT = DIRECT_;
    static constexpr int BM = BM_, BN = BN_, WM = WM_, WN = WN_, STAGES = STAGES_, BK = 128;
    static constexpr int KG = KG_, NW = WM * WN, NT = NW * 64 * KG, MI = BM / WM / 16, NI = BN / WN / 16;
    static constexpr int LA = BM / 8 / NW, LB = BN / 8 / NW, PER = LA + LB, STAGE = (BM + BN) * BK;
    static_assert(MI * WM * 16 == BM && NI * WN * 16 == BN && LA * 8 * NW == BM && LB * 8 * NW == BN && STAGES >= 2 && (DIRECT || STAGES == 2) && STAGE * STAGES * KG <= 160 * 1024 && NW * KG <= 16, "");
};

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

template <typename S>
__global__ __launch_bounds__(S::NT)
void product_tile(Product p)
{
    constexpr int BM = S::BM, BN = S::BN, BK = S::BK, MI = S::MI, NI = S::NI, LA = S::LA, LB = S::LB, PER = S::PER;
    __shared__ __attribute__((aligned(1024))) int8_t whole[S::KG * S::STAGES * S::STAGE];
    static_assert(S::NW * kPatch<float, NI> <= S::KG * S::STAGES * S::STAGE && (S::KG - 1) * S::NW * MI * NI * 1024 <= S::KG * S::STAGES * S::STAGE, "");
    Rows r;
    if (!find_rows(p, BM, row_tile(), &r)) return;
    const int tid = threadIdx.x, lane = tid & 63, all = uniform(tid >> 6), group = all / S::NW, wave = all % S::NW, wm = wave / S::WN, wn = wave % S::WN;
    const int n0 = blockIdx.x * BN;
    int8_t *const ring = whole + group * (S::STAGES * S::STAGE);
    i32x4 acc[MI][NI] = {};
    if (!r.zero) {
        const unsigned ring_at = uniform((int)(unsigned)(unsigned long)(__attribute__((address_space(3))) int8_t *)ring);
        // this wave's pieces of a slab: eight rows each, lane -> row lane / 8, chunk position lane % 8
        const int rows = (int)(r.last - r.first), cols = p.n - n0;
        unsigned off[PER];
#pragma unroll
        for (int t = 0; t < PER; ++t) {
            const bool is_a = t < LA;
            const int row = (is_a ? wave * LA + t : wave * LB + t - LA) * 8 + lane / 8, limit = is_a ? rows : cols;
            const int chunk = (lane & 7) ^ (row >> 1 & 7);
            off[t] = (unsigned)(row < limit ? row : limit - 1) * (unsigned)(is_a ? p.lda : p.ldb) + chunk * 16;
        }
        const int8_t *abase = uniform(p.a + r.first * p.lda), *bbase = uniform(p.b + ((long)r.expert * p.n + n0) * p.ldb);
        const int whole_slabs = p.k / BK, slabs = (p.k + BK - 1) / BK;
        const int steps = (slabs + S::KG - 1) / S::KG;      // of every group; a slab past the last one is zeros
        // This wave's share of a slab into a stage; a slab that K ends in, or that lies past it, is filled up with zeros.
        auto issue = [&](int step, int stage) {
            const int slab = step * S::KG + group;
            const int8_t *as = abase + (long)slab * BK, *bs = bbase + (long)slab * BK;
            const unsigned at = ring_at + stage * S::STAGE, at_a = at + wave * LA * 1024, at_b = at + BM * BK + wave * LB * 1024;
            if (slab < whole_slabs) {
#pragma unroll
                for (int t = 0; t < PER; ++t) load_to_lds(t < LA ? as : bs, off[t], t < LA ? at_a + t * 1024 : at_b + (t - LA) * 1024);
            } else {
#pragma unroll
                for (int t = 0; t < PER; ++t) {
                    const int row = (t < LA ? wave * LA + t : wave * LB + t - LA) * 8 + lane / 8, chunk = (lane & 7) ^ (row >> 1 & 7);
                    const unsigned to = t < LA ? at_a + t * 1024 : at_b + (t - LA) * 1024;
                    if (slab * BK + chunk * 16 < p.k) load_to_lds(t < LA ? as : bs, off[t], to);
                    else *(i32x4 *)(ring + (to - ring_at) + lane * 16) = i32x4{0, 0, 0, 0};
                }
            }
        };
        // The same by way of registers: fetch starts the loads, put stores what they brought.
        i32x4 hold[PER];
        auto fetch = [&](int step) {
            const int slab = step * S::KG + group;
            if (slab < whole_slabs) {
#pragma unroll
                for (int t = 0; t < PER; ++t) __builtin_memcpy(&hold[t], (t < LA ? abase : bbase) + (long)slab * BK + off[t], 16);
            } else {
#pragma unroll
                for (int t = 0; t < PER; ++t) {
                    const int row = (t < LA ? wave * LA + t : wave * LB + t - LA) * 8 + lane / 8, chunk = (lane & 7) ^ (row >> 1 & 7);
                    hold[t] = load_chunk((t < LA ? abase : bbase) + off[t] - chunk * 16, slab * BK + chunk * 16, p.k);
                }
            }
        };
        auto put = [&](int stage) {
#pragma unroll
            for (int t = 0; t < PER; ++t) *(i32x4 *)(ring + stage * S::STAGE + (t < LA ? (wave * LA + t) * 1024 : BM * BK + (wave * LB + t - LA) * 1024) + lane * 16) = hold[t];
        };
        // a stage that every wave has read is filled with the slab `step`
        auto refill = [&](int step, int stage) {
            if (S::DIRECT) issue(step, stage);
            else {
                put(stage);
                if (step + 1 < steps) fetch(step + 1);
            }
        };
        // this wave has read its part of a slab, and its part of the next one has landed
        auto wait_next = [&](bool more) {
            if (!S::DIRECT) WAIT_LGKM();
            else if (S::STAGES > 2 && more) WAIT_LGKM_VMCNT((S::STAGES - 2) * PER);
            else WAIT_LGKM_VMCNT(0);
        };
        // fragments: lane l holds row l % 16, the 16 values from 16 * (l / 16) of a step of 64
        const int sw = lane >> 1 & 7, fr = lane & 15;
        // prologue: slabs 0 .. STAGES - 1 under way, slab 0 landed, its first fragments read
        if (!S::DIRECT) fetch(0);
#pragma unroll
        for (int s = 0; s < S::STAGES; ++s)
            if (s < steps) refill(s, s);
        if (!S::DIRECT) WAIT_LGKM();
        else if (S::STAGES > 2 && steps > S::STAGES) WAIT_LGKM_VMCNT((S::STAGES - 1) * PER);
        else WAIT_LGKM_VMCNT(0);
        BARRIER();
        if constexpr (MI * NI <= 4) {
            // Few MFMAs a slab: reading a step's fragments takes longer than multiplying the step before.  The fragments of a whole slab are read at once, while the
            // slab before it is multiplied.
            i32x4 ag[2][2][MI], bg[2][2][NI];
            auto read_slab = [&](int set, int stage) {
#pragma unroll
                for (int kk = 0; kk < 2; ++kk) {
                    const int8_t *at = ring + stage * S::STAGE + (((kk * 4 + (lane >> 4)) ^ sw) << 4);
#pragma unroll
                    for (int i = 0; i < NI; ++i) bg[set][kk][i] = *(const i32x4 *)(at + BM * BK + (wn * NI * 16 + i * 16 + fr) * BK);
#pragma unroll
                    for (int i = 0; i < MI; ++i) ag[set][kk][i] = *(const i32x4 *)(at + (wm * MI * 16 + i * 16 + fr) * BK);
                }
            };
            read_slab(0, 0);
            int stage = 0;
            auto slab = [&](int q, int set) {
                const int next = stage + 1 == S::STAGES ? 0 : stage + 1;
                const bool more = q + S::STAGES < steps;
                wait_next(more);
                BARRIER();                  // every wave has read slab q, and slab q + 1 has landed
                read_slab(set ^ 1, next);
                if (more) refill(q + S::STAGES, stage);
                __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                for (int kk = 0; kk < 2; ++kk)
#pragma unroll
                    for (int m = 0; m < MI * NI; ++m)
                        acc[m / NI][m % NI] = __builtin_amdgcn_mfma_i32_16x16x64_i8(bg[set][kk][m % NI], ag[set][kk][m / NI], acc[m / NI][m % NI], 0, 0, 0);
                stage = next;
            };
            int q = 0;
            for (; q + 2 <= steps; q += 2) { slab(q, 0); slab(q + 1, 1); }
            if (q < steps) slab(q, 0);
        } else {
        i32x4 af[2][MI], bf[2][NI];
        auto read = [&](int buf, int stage, int kk, int i) {
            const int8_t *at = ring + stage * S::STAGE + (((kk * 4 + (lane >> 4)) ^ sw) << 4);
            if (i < NI) bf[buf][i] = *(const i32x4 *)(at + BM * BK + (wn * NI * 16 + i * 16 + fr) * BK);
            else af[buf][i - NI] = *(const i32x4 *)(at + (wm * MI * 16 + (i - NI) * 16 + fr) * BK);
        };
#pragma unroll
        for (int i = 0; i < MI + NI; ++i) read(0, 0, 0, i);
        // A slab in two steps of 64.  Between the MFMAs of the first the wave reads the second's fragments; behind the first MFMA of the second step every wave has
        // read the slab and the next one has landed: its first fragments are read and the stage is refilled.  (After the last slab the reads
        // fetch what the ring holds; nothing uses it.)
        int stage = 0;
        for (int q = 0; q < steps; ++q) {
            constexpr int SLOTS = MI * NI, NR = MI + NI;
            const int next = stage + 1 == S::STAGES ? 0 : stage + 1;
            const bool more = q + S::STAGES < steps;
#pragma unroll
            for (int kk = 0; kk < 2; ++kk) {
#pragma unroll
                for (int m = 0; m < SLOTS; ++m) {
                    acc[m / NI][m % NI] = __builtin_amdgcn_mfma_i32_16x16x64_i8(bf[kk][m % NI], af[kk][m / NI], acc[m / NI][m % NI], 0, 0, 0);
                    if (kk == 1 && m == 0) {
                        wait_next(more);
                        BARRIER();
                        if (more) refill(q + S::STAGES, stage);
                    }
                    const int lo = m * NR / SLOTS, hi = (m + 1) * NR / SLOTS;
#pragma unroll
                    for (int u = 0; u < NR / SLOTS + 1; ++u)
                        if (lo + u < hi) read(kk ^ 1, kk == 0 ? stage : next, kk ^ 1, lo + u);
                    __builtin_amdgcn_sched_barrier(0);
                }
            }
            stage = next;
        }
        }
        WAIT_LGKM_VMCNT(0);
    }
    __syncthreads();
    if (S::KG > 1) {                        // the groups' sums meet in LDS
        i32x4 *const sums = (i32x4 *)whole;
        if (group > 0)
#pragma unroll
            for (int i = 0; i < MI; ++i)
#pragma unroll
                for (int j = 0; j < NI; ++j) sums[((((group - 1) * S::NW + wave) * MI + i) * NI + j) * 64 + lane] = acc[i][j];
        __syncthreads();
        if (group == 0)
#pragma unroll
            for (int g = 0; g < S::KG - 1; ++g)
#pragma unroll
                for (int i = 0; i < MI; ++i)
#pragma unroll
                    for (int j = 0; j < NI; ++j) acc[i][j] += sums[(((g * S::NW + wave) * MI + i) * NI + j) * 64 + lane];
        __syncthreads();
        if (group > 0) return;
    }
    int8_t *const patch = whole + wave * kPatch<float, NI>;
    if (p.out == OPEVO_F32) store_tile<float>(p, r, wm * MI * 16, n0 + wn * NI * 16, acc, patch, lane);
    else if (p.out == OPEVO_BF16) store_tile<__bf16>(p, r, wm * MI * 16, n0 + wn * NI * 16, acc, patch, lane);
    else store_tile<_Float16>(p, r, wm * MI * 16, n0 + wn * NI * 16, acc, patch, lane);
}

using opevo::fail;

// How many tiles of bm rows there can be at most.  Grouped: each expert's last one is ragged, and so is that of the rows of none.
int64_t row_tiles(const Product &p, int bm) { return p.offsets ? std::min<int64_t>(p.m, p.m / bm + p.experts + 1) : (p.m + bm - 1) / bm; }

dim3 grid_of(const Product &p, int bm, int bn)
{
    const int64_t tiles = row_tiles(p, bm);
    return dim3((unsigned)((p.n + bn - 1) / bn), (unsigned)std::min<int64_t>(tiles, kGridY), (unsigned)((tiles + kGridY - 1) / kGridY));
}

template <typename S>
int run_tile(const Product &p, hipStream_t stream)
{
    return opevo::launch("product launch", product_tile<S>, grid_of(p, S::BM, S::BN), dim3(S::NT), stream, p);
}

template <int MI, int NI, int W>
int run_thin(const Product &p, hipStream_t stream)
{
    return opevo::launch("product launch", (product_thin<MI, NI, W>), grid_of(p, MI * 16, NI * 16), dim3(W * 64), stream, p);
}

// A kernel and what it takes, in us: launch + max(steps * chain, load * (tile + steps * rate)), where steps is how many slabs (thin: steps of 256 values) a wave
// goes through and load the workgroups for each of the 256 compute units, rounded up where that foretold the times better.  The first term is a workgroup's chain of latencies,
// the second what a compute unit gets through.  The constants were fitted to the times of every kernel at 400 (rows apart by multiples of 16) and 450 (others)
// random sizes of 1 - 8192 rows, 64 - 8192 columns and K of 64 - 8192; the kernel chosen by them took 0.8 % and 1.9 % more than the best of all of them in the
// geometric mean, at most 1.5 times as much.  All of these were plain products.  By experts the same constants are used with the tiles that an even deal of the rows would make;
// what a router deals makes more, and a ragged tile costs what a whole one does: 8192 rows over 8 experts, 34 - 37 tiles of 256 rows instead of 32, go in three rounds of
// workgroups instead of two and take 58 us where the plain product of that size (N 4096, K 1024) takes 42.
struct Kernel {
    int (*run)(const Product &, hipStream_t);
    int bm, bn, step, ways;             // tile, K of a step, waves or groups that share the steps
    int64_t most;                       // rows it is considered for
    bool round_up;
    float launch, chain, tile, rate;
};
constexpr int64_t kAll = INT64_MAX;
const Kernel kDirect[] = {
    {run_tile<Shape<true, 256, 256, 2, 4, 2>>, 256, 256, 128, 1, kAll, true, 0.f, 1.6f, 10.8f, 1.41f},
    {run_tile<Shape<true, 128, 128, 2, 4, 2>>, 128, 128, 128, 1, kAll, false, 3.03f, 0.844f, 2.47f, 0.66f},
    {run_tile<Shape<true, 128, 128, 2, 4, 4>>, 128, 128, 128, 1, kAll, true, 0.f, 0.f, 5.18f, 0.576f},
    {run_tile<Shape<true, 128, 64, 4, 2, 3>>, 128, 64, 128, 1, kAll, false, 2.76f, 0.383f, 1.24f, 0.544f},
    {run_tile<Shape<true, 64, 64, 2, 4, 4>>, 64, 64, 128, 1, kAll, false, 2.6f, 0.322f, 0.783f, 0.322f},
    {run_tile<Shape<true, 32, 128, 1, 4, 4>>, 32, 128, 128, 1, kAll, false, 2.92f, 0.269f, 0.802f, 0.431f},
    {run_tile<Shape<true, 32, 64, 1, 4, 4, 2>>, 32, 64, 128, 2, kAll, false, 2.72f, 0.371f, 1.27f, 0.462f},
    {run_tile<Shape<true, 32, 32, 2, 2, 6, 2>>, 32, 32, 128, 2, kAll, false, 2.39f, 0.26f, 0.532f, 0.372f},
    {run_thin<1, 1, 4>, 16, 16, 256, 4, 256, false, 2.22f, 0.683f, 0.f, 0.775f},
};
const Kernel kAny[] = {
    {run_tile<Shape<false, 128, 256, 2, 4, 2>>, 128, 256, 128, 1, kAll, true, 0.f, 0.f, 6.38f, 1.29f},
    {run_tile<Shape<false, 128, 128, 2, 4, 2>>, 128, 128, 128, 1, kAll, true, 0.f, 0.f, 4.32f, 0.78f},
    {run_tile<Shape<false, 128, 64, 4, 2, 2>>, 128, 64, 128, 1, kAll, true, 0.231f, 0.f, 3.27f, 0.597f},
    {run_tile<Shape<false, 64, 64, 2, 4, 2>>, 64, 64, 128, 1, kAll, true, 2.07f, 0.466f, 1.25f, 0.461f},
    {run_tile<Shape<false, 32, 64, 1, 4, 2, 2>>, 32, 64, 128, 2, kAll, true, 2.52f, 0.00958f, 1.04f, 0.569f},
    {run_tile<Shape<false, 32, 32, 2, 2, 2, 2>>, 32, 32, 128, 2, kAll, true, 2.4f, 0.545f, 0.501f, 0.363f},
    {run_tile<Shape<false, 32, 32, 2, 2, 2, 4>>, 32, 32, 128, 4, kAll, true, 1.51f, 0.864f, 1.59f, 0.678f},
    {run_thin<1, 1, 4>, 16, 16, 256, 4, 64, true, 0.993f, 2.07f, 0.f, 1.74f},
};

int run_product(const Product &p, hipStream_t stream)
{
    const auto whole = [](const void *at, long ld) { return reinterpret_cast<uintptr_t>(at) % 16 == 0 && ld % 16 == 0; };
    const bool direct = p.k % 16 == 0 && whole(p.a, p.lda) && whole(p.b, p.ldb);
    // a tile's rows are addressed by 32-bit offsets from its first
    const bool near = p.lda <= (1 << 24) && p.ldb <= (1 << 24);
    if (!near) return run_thin<1, 1, 4>(p, stream);
    // grouped: as if the rows were dealt evenly, which the host cannot know
    const int64_t parts = p.offsets ? std::min<int64_t>(p.experts, p.m) : 1, rows = (p.m + parts - 1) / parts;
    const Kernel *best = nullptr;
    float least = 0.f;
    const auto consider = [&](const Kernel &k) {
        if (rows > k.most) return;
        const int64_t groups = parts * ((rows + k.bm - 1) / k.bm) * ((p.n + k.bn - 1) / k.bn), slabs = (p.k + k.step - 1) / k.step;
        const float steps = (float)((slabs + k.ways - 1) / k.ways), load = k.round_up ? (float)((groups + 255) / 256) : (float)groups / 256.f;
        const float us = k.launch + std::max(steps * k.chain, load * (k.tile + steps * k.rate));
        if (!best || us < least) { best = &k; least = us; }
    };
    if (direct) for (const Kernel &k : kDirect) consider(k);
    else for (const Kernel &k : kAny) consider(k);
    return best->run(p, stream);
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
    return run_product(p, on);
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
