// Products of microscaled 4-bit numbers (mx4.hpp) along K:
//   C[m, n] = sum_k A[m, k] B[n, k],
// each operand the value of its code times the factor of its 32.  The matrix instruction takes the codes and the factors as they are stored (128 values and four factors a row at a time) and
// sums in fp32; the sum is rounded once to the output type.  B holds an output channel a row.  The grouped form gives each range of rows offsets[e] .. offsets[e + 1] a B of its own.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdint>
#include <type_traits>

#include "launch.hpp"
#include "mx4.hpp"
#include "narrow.hpp"
#include "product.hpp"
#include "rows.hpp"
#include "wave.hpp"

namespace {

typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

// What one call computes.  Plain: experts = 0, offsets = NULL.  Grouped: B has experts * N rows.
struct Product4 {
    const uint8_t *a, *b, *sa, *sb;
    long lda, ldb, ldsa, ldsb;
    const int *offsets;
    int experts;
    void *c;
    long ldc;
    int out;            // opevo_dtype
    long m;
    int n, k;           // k: bytes of a row, the last one half used where `odd`
    int blocks;         // factors of a row
    bool odd;
};

// Sixteen rows of either operand, 128 values: lane l holds 32 values of row l % 16 and their factor, in byte BYTE of its factor word.
template <int BYTE>
__device__ __forceinline__ f32x4 mfma(i32x4 b, i32x4 a, f32x4 c, int sb, int sa)
{
    const i32x8 b8 = {b[0], b[1], b[2], b[3], 0, 0, 0, 0}, a8 = {a[0], a[1], a[2], a[3], 0, 0, 0, 0};
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(b8, a8, c, 4, 4, BYTE, sb, BYTE, sa);
}
// The byte is known once the loops around are unrolled.
__device__ __forceinline__ f32x4 mfma_at(int byte, i32x4 b, i32x4 a, f32x4 c, int sb, int sa) { return byte ? mfma<1>(b, a, c, sb, sa) : mfma<0>(b, a, c, sb, sa); }

// Writes a wave's MI x NI atoms, rows r.first + m0 .. and columns col0 .. of C.  Lane l of an atom holds columns 4 * (l / 16) .. + 3 of row l % 16; the 16 rows of an atom row go through a
// piece of LDS of the wave's own and leave as whole lines, 16 bytes a lane.
template <typename T, int NI> constexpr int kPatch = 16 * NI * 16 * (int)sizeof(T);   // bytes of LDS a wave takes
template <typename T, int MI, int NI>
__device__ __forceinline__ void store_sums(const Product4 &p, const Rows &r, int m0, int col0, const f32x4 (&acc)[MI][NI], int8_t *patch, int lane)
{
    constexpr int PITCH = NI * 16 * (int)sizeof(T), CPR = NI * (int)sizeof(T), V = 16 / (int)sizeof(T);   // bytes, 16-byte chunks of a row, elements of a chunk
    static_assert((CPR & (CPR - 1)) == 0, "chunks are permuted by an exclusive or");
    const int cols = p.n - col0;
#pragma unroll
    for (int i = 0; i < MI; ++i) {
#pragma unroll
        for (int j = 0; j < NI; ++j) {
            T v[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] = narrow<T>(acc[i][j][e]);
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
            if (c + V <= cols) store_away(dst, __builtin_assume_aligned(from, 16));       // 8192 x 4096 x 1024 bf16 31.9 -> 29.3 us, 2048 rows 9.8 -> 8.0; as much less with a reader
            else
#pragma unroll 1
                for (int e = 0; e < cols - c; ++e) dst[e] = ((const T *)from)[e];
        }
        exchange();
    }
}

template <int MI, int NI>
__device__ __forceinline__ void store_as(const Product4 &p, const Rows &r, int m0, int col0, const f32x4 (&acc)[MI][NI], int8_t *patch, int lane)
{
    if (p.out == OPEVO_F32) store_sums<float>(p, r, m0, col0, acc, patch, lane);
    else if (p.out == OPEVO_BF16) store_sums<__bf16>(p, r, m0, col0, acc, patch, lane);
    else store_sums<_Float16>(p, r, m0, col0, acc, patch, lane);
}

// ------------------------------------------------------------------ few rows
// For few rows the weights are all there is to read, each once, and the time is that of one trip to memory.  Every wave loads its fragments and their factors from global memory into
// registers, 512 values along K a step (four MFMAs), the next step's while it multiplies.  The W waves of a workgroup share a tile of 16 x 16 and deal the steps among themselves;
// their sums meet in LDS.  Loads take any alignment.  1 x 4096 x 4096: 8.9 MB in 4.4 us, a launch and one trip to memory.
template <int W>
__global__ __launch_bounds__(W * 64)
void product4_thin(Product4 p)
{
    __shared__ f32x4 sums[W][64];
    Rows r;
    if (!find_rows(p, 16, row_tile(), &r)) return;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), n0 = blockIdx.x * 16, g = lane >> 4;
    f32x4 acc = {};
    if (!r.zero) {
        const long m = r.first + (lane & 15), ma = m < r.last ? m : r.last - 1, nb = (long)r.expert * p.n + min(n0 + (lane & 15), p.n - 1);
        const uint8_t *row[2] = {p.a + ma * p.lda, p.b + nb * p.ldb}, *by[2] = {p.sa + ma * p.ldsa, p.sb + nb * p.ldsb};
        const int steps = (p.k + 255) / 256;
        i32x4 v[2][4], w[2][4], fv[2], fw[2];
        auto load = [&](i32x4 (&to)[2][4], i32x4 (&f)[2], int step) {
            const int k0 = step * 256 + g * 16;
            if (step * 256 + 256 <= (p.odd ? p.k - 1 : p.k)) {
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    __builtin_memcpy(&f[i], by[i] + step * 16, 16);
#pragma unroll
                    for (int u = 0; u < 4; ++u) __builtin_memcpy(&to[i][u], row[i] + k0 + u * 64, 16);
                }
            } else {
                auto end = [&](auto is_long) __attribute__((always_inline)) {
#pragma unroll
                    for (int i = 0; i < 2; ++i)
#pragma unroll
                        for (int u = 0; u < 4; ++u) {
                            f[i][u] = load_factors<decltype(is_long)::value>(by[i], step * 16 + u * 4, p.blocks);
                            to[i][u] = load_codes<decltype(is_long)::value>(row[i], k0 + u * 64, p.k, p.odd);
                        }
                };
                if (p.blocks >= 4) end(std::true_type());
                else end(std::false_type());
            }
        };
        auto multiply = [&](const i32x4 (&of)[2][4], const i32x4 (&f)[2]) {
#pragma unroll
            for (int u = 0; u < 4; ++u) acc = mfma<0>(of[1][u], of[0][u], acc, (int)((unsigned)f[1][u] >> 8 * g), (int)((unsigned)f[0][u] >> 8 * g));
        };
        int s = wave;
        if (s < steps) load(v, fv, s);
        for (; s < steps; s += 2 * W) {
            if (s + W < steps) load(w, fw, s + W);
            multiply(v, fv);
            if (s + W >= steps) break;
            if (s + 2 * W < steps) load(v, fv, s + 2 * W);
            multiply(w, fw);
        }
    }
    sums[wave][lane] = acc;
    __syncthreads();
    if (wave > 0) return;
    f32x4 sum = sums[0][lane];
#pragma unroll
    for (int o = 1; o < W; ++o) sum += sums[o][lane];
    const long m = r.first + (lane & 15);
    if (m >= r.last) return;
    const float c[4] = {sum[0], sum[1], sum[2], sum[3]};
    const int col = n0 + g * 4;
    if (p.out == OPEVO_F32) store4((float *)p.c + m * p.ldc, col, p.n, c);
    else if (p.out == OPEVO_BF16) store4((__bf16 *)p.c + m * p.ldc, col, p.n, c);
    else store4((_Float16 *)p.c + m * p.ldc, col, p.n, c);
}

// ------------------------------------------------------------------ tiles
// Workgroup tile BM x BN, slabs of 128 bytes (256 values), WM x WN waves of MI x NI atoms of 16 x 16 x 128, KG groups of such waves that take every KG-th slab and add up
// their sums in LDS at the end.  The 16-byte chunk 2 g + kk of a row, which group g of lanes reads in step kk, sits at chunk position (g + 4 kk) ^ (row / 2 % 8) of its row of the slab: the lanes of
// a turn of a fragment read then fall on different groups of banks (with (2 g + kk) ^ ... half of the LDS cycles were conflicts).  Behind the rows of a slab stand their factors, eight bytes a row.  Rows past the end repeat the last one (their results are not stored); chunks past K are zeros.
// DIRECT: every wave issues wave-wide loads whose destination is LDS (16 bytes a lane for the codes, the chunk each lane loads chosen by the permutation, 4 for the factors); a
// ring of STAGES slabs keeps STAGES - 1 in flight.  For operands whose pointers and row lengths are multiples of 16 (factors: of 4) and K of 32.
// Otherwise the slabs pass through registers, from where they start on any address: two stages in LDS, the slab after them on its way.
// Many tiles: bound by the matrix pipes and by power (8192^3, 256 x 256: 278 us, 214 on zeros); few: by the chain of a workgroup's slabs, 0.3 - 1 us each, where groups help (333 rows by 24 experts x
// 1000 x 1001 12.2 us, 32 x 32 by way of registers).
template <bool DIRECT_, int BM_, int BN_, int WM_, int WN_, int STAGES_, int KG_ = 1>
struct Shape {
    static constexpr bool DIRECT = DIRECT_;
    static constexpr int BM = BM_, BN = BN_, WM = WM_, WN = WN_, STAGES = STAGES_, BK = 128;
    static constexpr int KG = KG_, NW = WM * WN, NT = NW * 64 * KG, MI = BM / WM / 16, NI = BN / WN / 16;
    static constexpr int LA = BM / 8 / NW, LB = BN / 8 / NW, PER = LA + LB, CODES = (BM + BN) * BK, STAGE = CODES + (BM + BN) * 8;
    static constexpr int FP = (BM + BN) / 32, FPER = (FP + NW - 1) / NW;      // pieces of 32 rows' factors, of a wave; pieces beyond the last one are loaded twice
    static constexpr int BYTES = KG * STAGES * STAGE;
    static_assert(MI * WM * 16 == BM && NI * WN * 16 == BN && LA * 8 * NW == BM && LB * 8 * NW == BN && BM % 32 == 0 && BN % 32 == 0 && STAGES >= 2 && (DIRECT || STAGES == 2)
                      && BYTES <= 160 * 1024 && NW * KG <= 16 && BM + BN <= NW * 64 && STAGE % 16 == 0,
                  "");
};

// The chunk at a position of a row.
__device__ __forceinline__ int chunk_for(int position, int row)
{
    const int at = position ^ (row >> 1 & 7);
    return (at & 3) << 1 | at >> 2;
}

// lane i's 4 bytes from base + off to LDS at lds + 4 i, as load_to_lds.
__device__ __forceinline__ void load_word_to_lds(const int8_t *base, unsigned off, unsigned lds)
{
    const int8_t *copy;
    asm volatile("s_mov_b32 m0, %3\n\ts_mov_b64 %0, %2\n\tglobal_load_lds_dword %1, %0" : "=&s"(copy) : "v"(off), "s"(base), "s"(lds) : "memory", "m0");
}

template <typename S>
__global__ __launch_bounds__(S::NT)
void product4_tile(Product4 p)
{
    constexpr int BM = S::BM, BN = S::BN, BK = S::BK, MI = S::MI, NI = S::NI, LA = S::LA, LB = S::LB, PER = S::PER, ALL = PER + S::FPER;
    __shared__ __attribute__((aligned(1024))) int8_t whole[S::BYTES];
    static_assert(S::NW * kPatch<float, NI> <= S::BYTES && (S::KG - 1) * S::NW * MI * NI * 1024 <= S::BYTES, "");
    Rows r;
    if (!find_rows(p, BM, row_tile(), &r)) return;
    const int tid = threadIdx.x, lane = tid & 63, all = uniform(tid >> 6), group = all / S::NW, wave = all % S::NW, wm = wave / S::WN, wn = wave % S::WN;
    const int n0 = blockIdx.x * BN;
    int8_t *const ring = whole + group * (S::STAGES * S::STAGE);
    f32x4 acc[MI][NI] = {};
    if (!r.zero) {
        const unsigned ring_at = uniform((int)(unsigned)(unsigned long)(__attribute__((address_space(3))) int8_t *)ring);
        // this wave's pieces of a slab: eight rows each, lane -> row lane / 8, chunk position lane % 8
        const int rows = (int)(r.last - r.first), cols = p.n - n0;
        unsigned off[PER];
#pragma unroll
        for (int t = 0; t < PER; ++t) {
            const bool is_a = t < LA;
            const int row = (is_a ? wave * LA + t : wave * LB + t - LA) * 8 + lane / 8, limit = is_a ? rows : cols;
            const int chunk = chunk_for(lane & 7, row);
            off[t] = (unsigned)(row < limit ? row : limit - 1) * (unsigned)(is_a ? p.lda : p.ldb) + chunk * 16;
        }
        const long b0 = (long)r.expert * p.n + n0;
        const int8_t *abase = uniform((const int8_t *)p.a + r.first * p.lda), *bbase = uniform((const int8_t *)p.b + b0 * p.ldb);
        const int8_t *afact = uniform((const int8_t *)p.sa + r.first * p.ldsa), *bfact = uniform((const int8_t *)p.sb + b0 * p.ldsb);
        // a row of the tile, A's before B's -> where its factors start
        auto factors_at = [&](int row) { return row < BM ? (unsigned)min(row, rows - 1) * (unsigned)p.ldsa : (unsigned)min(row - BM, cols - 1) * (unsigned)p.ldsb; };
        // and the wave's pieces of the factors: 32 rows each, lane -> row lane / 2, four of the eight factors
        unsigned foff[S::FPER];
        int fpiece[S::FPER];
#pragma unroll
        for (int t = 0; t < S::FPER; ++t) {
            fpiece[t] = (wave * S::FPER + t) % S::FP;
            foff[t] = factors_at(fpiece[t] * 32 + lane / 2) + (lane & 1) * 4;
        }
        const int whole_slabs = p.odd ? (p.k - 1) / BK : p.k / BK, slabs = (p.k + BK - 1) / BK;
        const int steps = (slabs + S::KG - 1) / S::KG;      // of every group; a slab past the last one is zeros
        // This wave's share of a slab into a stage: of a whole slab; of one that K ends in, or that lies past it, which is filled up with zeros.
        auto issue = [&](int step, int stage) {
            const int slab = step * S::KG + group;
            const int8_t *as = abase + (long)slab * BK, *bs = bbase + (long)slab * BK;
            const unsigned at = ring_at + stage * S::STAGE, at_a = at + wave * LA * 1024, at_b = at + BM * BK + wave * LB * 1024;
#pragma unroll
            for (int t = 0; t < PER; ++t) load_to_lds(t < LA ? as : bs, off[t], t < LA ? at_a + t * 1024 : at_b + (t - LA) * 1024);
#pragma unroll
            for (int t = 0; t < S::FPER; ++t) load_word_to_lds(uniform((fpiece[t] < BM / 32 ? afact : bfact) + (long)slab * 8), foff[t], at + S::CODES + fpiece[t] * 256);
        };
        auto issue_ragged = [&](int step, int stage) {
            const int slab = step * S::KG + group;
            const int8_t *as = abase + (long)slab * BK, *bs = bbase + (long)slab * BK;
            const unsigned at = ring_at + stage * S::STAGE, at_a = at + wave * LA * 1024, at_b = at + BM * BK + wave * LB * 1024;
#pragma unroll
            for (int t = 0; t < PER; ++t) {
                const int row = (t < LA ? wave * LA + t : wave * LB + t - LA) * 8 + lane / 8, chunk = chunk_for(lane & 7, row);
                const unsigned to = t < LA ? at_a + t * 1024 : at_b + (t - LA) * 1024;
                if (slab * BK + chunk * 16 < p.k) load_to_lds(t < LA ? as : bs, off[t], to);
                else *(i32x4 *)(ring + (to - ring_at) + lane * 16) = i32x4{0, 0, 0, 0};
            }
#pragma unroll
            for (int t = 0; t < S::FPER; ++t) {
                const uint8_t *of = (const uint8_t *)(fpiece[t] < BM / 32 ? afact : bfact) + (foff[t] - (lane & 1) * 4);
                const int b = slab * 8 + (lane & 1) * 4;
                *(int *)(ring + stage * S::STAGE + S::CODES + fpiece[t] * 256 + lane * 4) = p.blocks >= 4 ? load_factors<true>(of, b, p.blocks) : load_factors<false>(of, b, p.blocks);
            }
        };
        // The same by way of registers: fetch starts the loads, put stores what they brought.  A thread takes the factors of one row.
        i32x4 hold[PER];
        int fhold[2];
        const int mine = (wave * 64 + lane) % (BM + BN);      // threads beyond the last row take one again
        auto fetch = [&](int step) {
            const int slab = step * S::KG + group;
#pragma unroll
            for (int t = 0; t < PER; ++t) __builtin_memcpy(&hold[t], (t < LA ? abase : bbase) + (long)slab * BK + off[t], 16);
            __builtin_memcpy(fhold, (mine < BM ? afact : bfact) + factors_at(mine) + (long)slab * 8, 8);
        };
        auto fetch_end = [&](auto is_long, int step) __attribute__((always_inline)) {
            constexpr bool LONG = decltype(is_long)::value;
            const int slab = step * S::KG + group;
#pragma unroll
            for (int t = 0; t < PER; ++t) {
                const int row = (t < LA ? wave * LA + t : wave * LB + t - LA) * 8 + lane / 8, chunk = chunk_for(lane & 7, row);
                hold[t] = load_codes<LONG>((const uint8_t *)(t < LA ? abase : bbase) + off[t] - chunk * 16, slab * BK + chunk * 16, p.k, p.odd);
            }
            const uint8_t *of = (const uint8_t *)(mine < BM ? afact : bfact) + factors_at(mine);
            fhold[0] = load_factors<LONG>(of, slab * 8, p.blocks);
            fhold[1] = load_factors<LONG>(of, slab * 8 + 4, p.blocks);
        };
        auto fetch_ragged = [&](int step) __attribute__((always_inline)) {
            if (p.blocks >= 4) fetch_end(std::true_type(), step);
            else fetch_end(std::false_type(), step);
        };
        auto put = [&](int stage) {
#pragma unroll
            for (int t = 0; t < PER; ++t) *(i32x4 *)(ring + stage * S::STAGE + (t < LA ? (wave * LA + t) * 1024 : BM * BK + (wave * LB + t - LA) * 1024) + lane * 16) = hold[t];
            __builtin_memcpy(__builtin_assume_aligned(ring + stage * S::STAGE + S::CODES + mine * 8, 8), fhold, 8);
        };
        // A stage that every wave has read is filled with the slab `step`, if there is one.  HOW says what has to be loaded for that: a whole slab, anything or nothing.  The loop over slabs is
        // three, one for each, because a branch among a slab's MFMAs has the compiler move them behind it (256 x 256: all reads, then all MFMAs, and spills).
        enum How { kWhole, kAny, kNone };
        auto is_whole = [&](int step) { return step * S::KG + group < whole_slabs; };
        auto refill = [&](auto how, int step, int stage) {
            constexpr How HOW = decltype(how)::value;
            if constexpr (S::DIRECT) {
                if constexpr (HOW == kWhole) issue(step, stage);
                else if constexpr (HOW == kAny) {
                    if (step < steps) {
                        if (is_whole(step)) issue(step, stage);
                        else issue_ragged(step, stage);
                    }
                }
            } else {
                if constexpr (HOW != kNone) put(stage);
                if constexpr (HOW == kWhole) fetch(step + 1);
                else if constexpr (HOW == kAny) {
                    if (step + 1 < steps) {
                        if (is_whole(step + 1)) fetch(step + 1);
                        else fetch_ragged(step + 1);
                    }
                }
            }
        };
        using Whole = std::integral_constant<How, kWhole>;
        using Any = std::integral_constant<How, kAny>;
        using None = std::integral_constant<How, kNone>;
        // the slab whose load slab q sets off
        constexpr int AHEAD = S::DIRECT ? S::STAGES : S::STAGES + 1;
        // this wave has read its part of a slab, and its part of the next one has landed
        auto wait_next = [&](bool more) {
            if (!S::DIRECT) WAIT_LGKM();
            else if (S::STAGES > 2 && more) WAIT_LGKM_VMCNT((S::STAGES - 2) * ALL);
            else WAIT_LGKM_VMCNT(0);
        };
        // fragments: lane l holds row l % 16, and of the step kk the 32 values from 64 * (l / 16) + 32 kk on; both steps' factors in a word
        const int sw = lane >> 1 & 7, fr = lane & 15, g = lane >> 4;
        auto chunk_at = [&](int stage, int kk) { return ring + stage * S::STAGE + ((g + 4 * kk ^ sw) << 4); };
        auto read_factor = [&](int stage, int row) { return (int)*(const uint16_t *)(ring + stage * S::STAGE + S::CODES + (row + fr) * 8 + g * 2); };
        // prologue: slabs 0 .. STAGES - 1 under way, slab 0 landed, its first fragments read
        if (!S::DIRECT) {
            if (is_whole(0)) fetch(0);
            else fetch_ragged(0);
        }
#pragma unroll
        for (int s = 0; s < S::STAGES; ++s)
            if (s < steps) refill(Any(), s, s);
        if (!S::DIRECT) WAIT_LGKM();
        else if (S::STAGES > 2 && steps > S::STAGES) WAIT_LGKM_VMCNT((S::STAGES - 1) * ALL);
        else WAIT_LGKM_VMCNT(0);
        BARRIER();
        if constexpr (MI * NI <= 4) {
            // Few MFMAs a slab: the fragments of a whole slab are read at once, while the slab before it is multiplied.
            i32x4 ag[2][2][MI], bg[2][2][NI];
            int fa[2][MI], fb[2][NI];
            auto read_slab = [&](int set, int stage) {
#pragma unroll
                for (int i = 0; i < MI; ++i) fa[set][i] = read_factor(stage, (wm * MI + i) * 16);
#pragma unroll
                for (int i = 0; i < NI; ++i) fb[set][i] = read_factor(stage, BM + (wn * NI + i) * 16);
#pragma unroll
                for (int kk = 0; kk < 2; ++kk) {
                    const int8_t *at = chunk_at(stage, kk);
#pragma unroll
                    for (int i = 0; i < NI; ++i) bg[set][kk][i] = *(const i32x4 *)(at + BM * BK + (wn * NI * 16 + i * 16 + fr) * BK);
#pragma unroll
                    for (int i = 0; i < MI; ++i) ag[set][kk][i] = *(const i32x4 *)(at + (wm * MI * 16 + i * 16 + fr) * BK);
                }
            };
            read_slab(0, 0);
            int stage = 0;
            auto slab = [&](auto how, int q, int set) {
                const int next = stage + 1 == S::STAGES ? 0 : stage + 1;
                const bool more = q + S::STAGES < steps;
                wait_next(more);
                BARRIER();                  // every wave has read slab q, and slab q + 1 has landed
                read_slab(set ^ 1, next);
                refill(how, q + S::STAGES, stage);
                __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                for (int kk = 0; kk < 2; ++kk)
#pragma unroll
                    for (int m = 0; m < MI * NI; ++m) {
                        const int i = m / NI, j = m % NI;
                        acc[i][j] = mfma_at(kk, bg[set][kk][j], ag[set][kk][i], acc[i][j], fb[set][j], fa[set][i]);
                    }
                stage = next;
            };
            int q = 0;
            for (; is_whole(q + 1 + AHEAD); q += 2) { slab(Whole(), q, 0); slab(Whole(), q + 1, 1); }
            for (; q + S::STAGES < steps; q += 2) {
                slab(Any(), q, 0);
                if (q + 1 < steps) slab(Any(), q + 1, 1);
            }
            for (; q < steps; q += 2) {
                slab(None(), q, 0);
                if (q + 1 < steps) slab(None(), q + 1, 1);
            }
        } else {
        // A slab is 2 MI fragments of A, those of its first 128 values before the others, each multiplied by the NI of B.  The one that comes D fragments later is read meanwhile, into
        // one of R places: holding both steps' fragments of a 256 x 256 tile would take more registers than there are.
        constexpr int D = MI == 8 ? 3 : MI, R = MI == 8 ? 4 : 2 * MI, LAST = 2 * MI - D;
        static_assert(2 * MI % R == 0 && D < R && LAST >= MI && MI >= NI && D * NI > NI, "");
        i32x4 af[R], bf[2][NI];
        int fa[MI], fb[NI], fb_next[NI];    // A's are read for the next slab as this one is done with them, B's are needed to its end
        auto read_a = [&](int stage, int f) { af[f % R] = *(const i32x4 *)(chunk_at(stage, f / MI) + (wm * MI * 16 + f % MI * 16 + fr) * BK); };
        auto read_b = [&](int stage, int kk, int i) { bf[kk][i] = *(const i32x4 *)(chunk_at(stage, kk) + BM * BK + (wn * NI * 16 + i * 16 + fr) * BK); };
        auto read_fa = [&](int stage, int i) { fa[i] = read_factor(stage, (wm * MI + i) * 16); };
        auto read_fb = [&](int (&to)[NI], int stage) {
#pragma unroll
            for (int i = 0; i < NI; ++i) to[i] = read_factor(stage, BM + (wn * NI + i) * 16);
        };
#pragma unroll
        for (int i = 0; i < NI; ++i) read_b(0, 0, i);
#pragma unroll
        for (int f = 0; f < D; ++f) read_a(0, f);
#pragma unroll
        for (int i = 0; i < MI; ++i) read_fa(0, i);
        read_fb(fb, 0);
        // Behind the first MFMA of fragment LAST every wave has read the slab and the next one has landed: its factors and first fragments are read and the stage is refilled.  (After
        // the last slab the reads fetch what the ring holds; nothing uses it.)
        int stage = 0;
        auto slab = [&](auto how, int q) {
            const int next = stage + 1 == S::STAGES ? 0 : stage + 1;
            const bool more = q + S::STAGES < steps;
#pragma unroll
            for (int f = 0; f < 2 * MI; ++f) {
                const int kk = f / MI, x = f % MI;
#pragma unroll
                for (int y = 0; y < NI; ++y) {
                    acc[x][y] = mfma_at(kk, bf[kk][y], af[f % R], acc[x][y], fb[y], fa[x]);
                    if (f == LAST && y == 0) {
                        wait_next(more);
                        BARRIER();
                        read_fb(fb_next, next);
                        if constexpr (decltype(how)::value == kWhole) refill(how, q + S::STAGES, stage);
                    }
                    if (y == 0) read_a(f + D < 2 * MI ? stage : next, (f + D) % (2 * MI));
                    if (y == 1 && f < NI) read_b(stage, 1, f);
                    const int past = (f - LAST) * NI + y - 1;
                    if (past >= 0 && past < NI) read_b(next, 0, past);
                    if (f >= LAST && y == NI - 1)
#pragma unroll
                        for (int i = f == LAST ? 0 : x; i <= x; ++i) read_fa(next, i);
                    __builtin_amdgcn_sched_barrier(0);
                }
            }
#pragma unroll
            for (int i = 0; i < NI; ++i) fb[i] = fb_next[i];
            if constexpr (decltype(how)::value == kAny) {
#pragma unroll
                for (int m = 0; m < MI * NI; ++m) asm volatile("" : "+v"(acc[m / NI][m % NI]));      // the sums are due here
                refill(how, q + S::STAGES, stage);
            }
            stage = next;
        };
        int q = 0;
        for (; is_whole(q + AHEAD); ++q) slab(Whole(), q);
        for (; q + S::STAGES < steps; ++q) slab(Any(), q);
        for (; q < steps; ++q) slab(None(), q);
        }
        WAIT_LGKM_VMCNT(0);
    }
    __syncthreads();
    if (S::KG > 1) {                        // the groups' sums meet in LDS
        f32x4 *const sums = (f32x4 *)whole;
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
    store_as(p, r, wm * MI * 16, n0 + wn * NI * 16, acc, whole + wave * kPatch<float, NI>, lane);
}

// ------------------------------------------------------------------ tiles of long rows
// The same for operands that can come straight to LDS and whose K is a multiple of 1024, so that nothing is ragged.  The factors come for four slabs at a time, 32 bytes a row, two sets in turn:
// eight bytes a row with every slab take as many requests as the codes, and cost 8192^3 some 40 us.  A set stands as two halves of [rows][16] bytes, each for two slabs.
// 8192^3, 256 x 256: 238 - 250 us (4.4 - 4.6 PFLOP/s), matrix pipes 59 % busy.  The instruction alone, from registers, makes 6.7 PFLOP/s of random codes and 9.4 of zeros; on zeros the kernel takes
// 196 - 206 us where that would be 117: power is a part of what it lacks, waits for LDS and barriers (34 % of the waves' time) the other.
// Factors start on multiples of 4 bytes: 16-byte loads take those.
template <int BM_, int BN_, int WM_, int WN_, int STAGES_>
struct LongShape {
    static constexpr int BM = BM_, BN = BN_, WM = WM_, WN = WN_, STAGES = STAGES_, BK = 128, ROWS = BM + BN;
    static constexpr int NW = WM * WN, NT = NW * 64, MI = BM / WM / 16, NI = BN / WN / 16;
    static constexpr int LA = BM / 8 / NW, LB = BN / 8 / NW, PER = LA + LB, STAGE = ROWS * BK;
    static constexpr int SET = ROWS * 32, PIECES = ROWS * 2 / 64, FPER = PIECES / NW, BYTES = STAGES * STAGE + 2 * SET;
    // two slabs at least lie between a set's loads and its first use, and no more than two slabs' loads are on their way behind them when they are waited for
    static_assert(MI * WM * 16 == BM && NI * WN * 16 == BN && LA * 8 * NW == BM && LB * 8 * NW == BN && FPER * NW == PIECES && BM % 64 == 0 && (STAGES == 2 || STAGES == 4) && MI >= NI
                      && BYTES <= 160 * 1024 && NW * kPatch<float, NI> <= BYTES,
                  "");
};

#define LDS(T) const __attribute__((address_space(3))) T *
template <typename S>
__global__ __launch_bounds__(S::NT)
void product4_long(Product4 p)
{
    constexpr int BM = S::BM, BN = S::BN, BK = S::BK, MI = S::MI, NI = S::NI, LA = S::LA, LB = S::LB, PER = S::PER, ROWS = S::ROWS;
    __shared__ __attribute__((aligned(1024))) int8_t ring[S::BYTES];
    Rows r;
    if (!find_rows(p, BM, row_tile(), &r)) return;
    r.first = (long)uniform((const int8_t *)r.first);           // alike for all lanes, which the compiler does not see: they would take vector registers to the end
    r.last = (long)uniform((const int8_t *)r.last);
    const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6), wm = wave / S::WN, wn = wave % S::WN, n0 = blockIdx.x * BN;
    f32x4 acc[MI][NI] = {};
    if (!r.zero) {
        const unsigned ring_at = uniform((int)(unsigned)(unsigned long)(__attribute__((address_space(3))) int8_t *)ring), sets_at = ring_at + S::STAGES * S::STAGE;
        const int rows = (int)(r.last - r.first), cols = p.n - n0, steps = p.k / BK;
        const long b0 = (long)r.expert * p.n + n0;
        // this wave's pieces of a slab: eight rows each, lane -> row lane / 8, chunk position lane % 8; and of a set: 64 rows of a half each
        unsigned off[PER], foff[S::FPER];
#pragma unroll
        for (int t = 0; t < PER; ++t) {
            const bool is_a = t < LA;
            const int row = (is_a ? wave * LA + t : wave * LB + t - LA) * 8 + lane / 8;
            off[t] = (unsigned)min(row, (is_a ? rows : cols) - 1) * (unsigned)(is_a ? p.lda : p.ldb);
            asm("" : "+v"(off[t]));         // product and sum in one instruction would take, and keep, two registers
            off[t] += chunk_for(lane & 7, row) * 16;
        }
        int half[S::FPER], first[S::FPER];
#pragma unroll
        for (int t = 0; t < S::FPER; ++t) {
            const int piece = wave * S::FPER + t, row = piece % (ROWS / 64) * 64 + lane;
            half[t] = piece / (ROWS / 64);
            first[t] = piece % (ROWS / 64) * 64;
            foff[t] = first[t] < BM ? (unsigned)min(row, rows - 1) * (unsigned)p.ldsa : (unsigned)min(row - BM, cols - 1) * (unsigned)p.ldsb;
        }
        const int8_t *abase = uniform((const int8_t *)p.a + r.first * p.lda), *bbase = uniform((const int8_t *)p.b + b0 * p.ldb);
        const int8_t *afact = uniform((const int8_t *)p.sa + r.first * p.ldsa), *bfact = uniform((const int8_t *)p.sb + b0 * p.ldsb);
        auto issue = [&](int step, int stage) {
            const int8_t *as = abase + (long)step * BK, *bs = bbase + (long)step * BK;
            const unsigned at = ring_at + stage * S::STAGE, at_a = at + wave * LA * 1024, at_b = at + BM * BK + wave * LB * 1024;
#pragma unroll
            for (int t = 0; t < PER; ++t) load_to_lds(t < LA ? as : bs, off[t], t < LA ? at_a + t * 1024 : at_b + (t - LA) * 1024);
        };
        // Nothing counts these loads: waits for so many slabs in flight wait for them as well, as they are older.
        auto issue_set = [&](int set) {
#pragma unroll
            for (int t = 0; t < S::FPER; ++t)
                load_to_lds(uniform((first[t] < BM ? afact : bfact) + (long)set * 32 + half[t] * 16), foff[t], sets_at + (set & 1) * S::SET + half[t] * (ROWS * 16) + first[t] * 16);
        };
        // fragments: lane l holds row l % 16, and of the step kk the 32 values from 64 * (l / 16) + 32 kk on; both steps' factors in a word
        constexpr int D = MI == 8 ? 3 : MI, R = MI == 8 ? 4 : 2 * MI, LAST = 2 * MI - D;
        static_assert(2 * MI % R == 0 && D < R && LAST >= MI && D * NI > NI, "");
        // Where they stand, as LDS addresses that go on from slab to slab: A's and B's of either step, and the factors.
        static_assert((S::STAGES & (S::STAGES - 1)) == 0 && (S::STAGE & (S::STAGE - 1)) == 0 && (S::SET & (S::SET - 1)) == 0, "stages and sets differ in a bit of the address");
        const int sw = lane >> 1 & 7, fr = lane & 15, g = lane >> 4;
        unsigned at_a[2], at_b[2], at_fa = sets_at + (wm * MI * 16 + fr) * 16 + g * 2, at_fb = sets_at + (BM + wn * NI * 16 + fr) * 16 + g * 2;
#pragma unroll
        for (int kk = 0; kk < 2; ++kk) {
            at_a[kk] = ring_at + (wm * MI * 16 + fr) * BK + ((g + 4 * kk ^ sw) << 4);
            at_b[kk] = ring_at + (BM + wn * NI * 16 + fr) * BK + ((g + 4 * kk ^ sw) << 4);
        }
        i32x4 af[R], bf[2][NI];
        int fa[MI], fb[2][NI];
        auto read_a = [&](int f) { af[f % R] = *(LDS(i32x4))(at_a[f / MI] + f % MI * 16 * BK); };
        auto read_b = [&](int kk, int i) { bf[kk][i] = *(LDS(i32x4))(at_b[kk] + i * 16 * BK); };
        auto factor_at = [&](unsigned at, int j, int i) { return (int)*(LDS(uint16_t))(at + j / 2 * (ROWS * 16) + j % 2 * 8 + i * 256); };
        issue_set(0);
#pragma unroll
        for (int s = 0; s < S::STAGES; ++s) issue(s, s);        // there are four slabs at least
        if (S::STAGES > 2) WAIT_LGKM_VMCNT((S::STAGES - 1) * PER);
        else WAIT_LGKM_VMCNT(0);
        BARRIER();
#pragma unroll
        for (int i = 0; i < NI; ++i) read_b(0, i);
#pragma unroll
        for (int f = 0; f < D; ++f) read_a(f);
#pragma unroll
        for (int i = 0; i < MI; ++i) fa[i] = factor_at(at_fa, 0, i);
#pragma unroll
        for (int i = 0; i < NI; ++i) fb[0][i] = factor_at(at_fb, 0, i);
        // Slab j of a set, as in product4_tile.
        auto slab = [&](auto at, auto last, int q) {
            constexpr int J = decltype(at)::value;
            constexpr bool MORE = !decltype(last)::value || J < 3, REFILL = !decltype(last)::value || J + S::STAGES < 4, AFTER = !decltype(last)::value || J + S::STAGES - 1 < 4;
#pragma unroll
            for (int f = 0; f < 2 * MI; ++f) {
                const int kk = f / MI, x = f % MI;
#pragma unroll
                for (int y = 0; y < NI; ++y) {
                    acc[x][y] = mfma_at(kk, bf[kk][y], af[f % R], acc[x][y], fb[J & 1][y], fa[x]);
                    if (MORE && f == LAST && y == 0) {
                        if (S::STAGES > 2 && AFTER) WAIT_LGKM_VMCNT((S::STAGES - 2) * PER);
                        else WAIT_LGKM_VMCNT(0);
                        BARRIER();
                        // on to the next stage, and set (the compiler is not to keep an address for each)
                        constexpr unsigned flip = ((J + 1) % S::STAGES ^ J % S::STAGES) * S::STAGE;
#pragma unroll
                        for (int o = 0; o < 2; ++o) {
                            at_a[o] ^= flip;
                            at_b[o] ^= flip;
                            asm("" : "+v"(at_a[o]), "+v"(at_b[o]));
                        }
                        if (J == 3) {
                            at_fa ^= S::SET;
                            at_fb ^= S::SET;
                        }
                        asm("" : "+v"(at_fa), "+v"(at_fb));
#pragma unroll
                        for (int i = 0; i < NI; ++i) fb[(J + 1) & 1][i] = factor_at(at_fb, (J + 1) % 4, i);
                        if constexpr (REFILL) issue(q + J + S::STAGES, J % S::STAGES);
                        if constexpr (J == 0 && !decltype(last)::value) issue_set(q / 4 + 1);
                    }
                    if (y == 0 && (MORE || f + D < 2 * MI)) read_a((f + D) % (2 * MI));
                    if (y == 1 && f < NI) read_b(1, f);
                    const int past = (f - LAST) * NI + y - 1;
                    if (MORE && past >= 0 && past < NI) read_b(0, past);
                    if (MORE && f >= LAST && y == NI - 1)
#pragma unroll
                        for (int i = f == LAST ? 0 : x; i <= x; ++i) fa[i] = factor_at(at_fa, (J + 1) % 4, i);
                    __builtin_amdgcn_sched_barrier(0);
                }
            }
        };
        auto four = [&](auto last, int q) {
            slab(std::integral_constant<int, 0>(), last, q);
            slab(std::integral_constant<int, 1>(), last, q);
            slab(std::integral_constant<int, 2>(), last, q);
            slab(std::integral_constant<int, 3>(), last, q);
        };
        int q = 0;
        for (; q + 4 < steps; q += 4) four(std::false_type(), q);
        four(std::true_type(), q);
        WAIT_LGKM_VMCNT(0);
    }
    __syncthreads();
    store_as(p, r, wm * MI * 16, n0 + wn * NI * 16, acc, ring + wave * kPatch<float, NI>, lane);
}


using opevo::launch;

// How many tiles of bm rows there can be at most.  Grouped: each expert's last one is ragged, and so is that of the rows of none.
int64_t row_tiles(const Product4 &p, int bm) { return p.offsets ? std::min<int64_t>(p.m, p.m / bm + p.experts + 1) : (p.m + bm - 1) / bm; }

dim3 grid_of(const Product4 &p, int bm, int bn)
{
    const int64_t tiles = row_tiles(p, bm);
    return dim3((unsigned)((p.n + bn - 1) / bn), (unsigned)std::min<int64_t>(tiles, kGridY), (unsigned)((tiles + kGridY - 1) / kGridY));
}

template <typename S>
int run_tile(const Product4 &p, hipStream_t stream)
{
    return launch("product4 launch", product4_tile<S>, grid_of(p, S::BM, S::BN), dim3(S::NT), stream, p);
}

template <typename S>
int run_long(const Product4 &p, hipStream_t stream)
{
    return launch("product4 launch", product4_long<S>, grid_of(p, S::BM, S::BN), dim3(S::NT), stream, p);
}

template <int W>
int run_thin(const Product4 &p, hipStream_t stream)
{
    return launch("product4 launch", product4_thin<W>, grid_of(p, 16, 16), dim3(W * 64), stream, p);
}

// A kernel and what it takes, in us: launch + max(steps * chain, load * (tile + steps * rate)), where steps is how many slabs (thin: steps of 256 bytes) a wave
// goes through and load the workgroups for each of the 256 compute units, rounded up where that foretold the times better.  The first term is a workgroup's chain of latencies,
// the second what a compute unit gets through.  The constants were fitted to the times of every kernel at 750 random sizes of 1 - 8192 rows, 64 - 8192 columns and K of 64 - 8192 (a third
// each of K in multiples of 1024, of 32, and any), those near the best one's counting most; the kernel chosen by them took 2.3, 2.8 and 1.7 % more than the best of all
// in the geometric mean, at most 1.9 times as much.  By experts they are used with the tiles that an even deal of the rows would make.
struct Kernel {
    int (*run)(const Product4 &, hipStream_t);
    int bm, bn, step, ways;             // tile, bytes of a step, waves or groups that share the steps
    int64_t most;                       // rows it is considered for
    bool round_up;
    float launch, chain, tile, rate;
};
constexpr int64_t kAll = INT64_MAX;
const Kernel kLong[] = {                // besides those of kDirect
    {run_long<LongShape<256, 256, 2, 4, 2>>, 256, 256, 128, 1, kAll, false, 6.78f, 1.38f, 8.53f, 2.33f},
    {run_long<LongShape<128, 128, 2, 2, 2>>, 128, 128, 128, 1, kAll, false, 4.18f, 0.591f, 1.22f, 0.822f},
    {run_long<LongShape<128, 128, 2, 4, 4>>, 128, 128, 128, 1, kAll, false, 3.63f, 0.583f, 2.34f, 0.922f},
};
const Kernel kDirect[] = {
    {run_tile<Shape<true, 256, 256, 2, 4, 2>>, 256, 256, 128, 1, kAll, false, 6.14f, 1.76f, 9.48f, 2.71f},
    {run_tile<Shape<true, 128, 128, 2, 2, 2>>, 128, 128, 128, 1, kAll, false, 4.36f, 0.97f, 2.06f, 0.939f},
    {run_tile<Shape<true, 128, 128, 2, 4, 4>>, 128, 128, 128, 1, kAll, false, 3.95f, 0.751f, 2.98f, 1.07f},
    {run_tile<Shape<true, 128, 64, 4, 2, 3>>, 128, 64, 128, 1, kAll, true, 1.4f, 0.34f, 2.43f, 0.562f},
    {run_tile<Shape<true, 64, 64, 2, 2, 4>>, 64, 64, 128, 1, kAll, false, 3.78f, 0.279f, 0.594f, 0.383f},
    {run_tile<Shape<true, 32, 64, 1, 4, 4, 2>>, 32, 64, 128, 2, kAll, false, 3.58f, 0.409f, 1.22f, 0.688f},
    {run_tile<Shape<true, 32, 32, 2, 2, 6, 2>>, 32, 32, 128, 2, kAll, true, 1.66f, 0.432f, 1.84f, 0.337f},
    {run_thin<4>, 16, 16, 256, 4, 300, true, 2.53f, 0.801f, 0.f, 0.667f},
};
const Kernel kAny[] = {
    {run_tile<Shape<false, 128, 128, 2, 4, 2>>, 128, 128, 128, 1, kAll, true, 0.634f, 1.42f, 4.16f, 1.21f},
    {run_tile<Shape<false, 128, 64, 4, 2, 2>>, 128, 64, 128, 1, kAll, true, 1.36f, 1.04f, 3.07f, 0.891f},
    {run_tile<Shape<false, 64, 64, 2, 4, 2>>, 64, 64, 128, 1, kAll, false, 4.05f, 0.479f, 1.28f, 0.846f},
    {run_tile<Shape<false, 32, 64, 1, 4, 2, 2>>, 32, 64, 128, 2, kAll, true, 1.6f, 0.039f, 2.74f, 0.737f},
    {run_tile<Shape<false, 32, 32, 2, 2, 2, 2>>, 32, 32, 128, 2, kAll, true, 3.05f, 0.543f, 0.804f, 0.49f},
    {run_thin<4>, 16, 16, 256, 4, 300, true, 2.18f, 2.f, 0.f, 1.12f},
};

int run_product4(const Product4 &p, hipStream_t stream)
{
    const auto whole = [](const void *at, long ld, int to) { return reinterpret_cast<uintptr_t>(at) % to == 0 && ld % to == 0; };
    const bool direct = p.k % 16 == 0 && !p.odd && whole(p.a, p.lda, 16) && whole(p.b, p.ldb, 16) && whole(p.sa, p.ldsa, 4) && whole(p.sb, p.ldsb, 4);
    // a tile's rows are addressed by 32-bit offsets from its first
    constexpr long kNear = 1 << 24;
    if (p.lda > kNear || p.ldb > kNear || p.ldsa > kNear || p.ldsb > kNear) return run_thin<4>(p, stream);
    // grouped: as if the rows were dealt evenly, which the host cannot know
    const int64_t parts = p.offsets ? std::min<int64_t>(p.experts, p.m) : 1, rows = (p.m + parts - 1) / parts;
    const Kernel *best = nullptr;
    float least = 0.f;
    const auto consider = [&](const Kernel &k) {
        if (rows > k.most) return;
        // experts' rows end anywhere in a tile: half a tile more each
        const float down = p.offsets ? parts * std::max(1.f, (float)rows / k.bm + 0.5f) : (float)((rows + k.bm - 1) / k.bm), groups = down * (float)((p.n + k.bn - 1) / k.bn);
        const int64_t slabs = (p.k + k.step - 1) / k.step;
        const float steps = (float)((slabs + k.ways - 1) / k.ways), load = k.round_up ? std::ceil(groups / 256.f) : groups / 256.f;
        const float us = k.launch + std::max(steps * k.chain, load * (k.tile + steps * k.rate));
        if (!best || us < least) { best = &k; least = us; }
    };
    if (direct && p.k % (4 * 128) == 0) for (const Kernel &k : kLong) consider(k);
    if (direct) for (const Kernel &k : kDirect) consider(k);
    else for (const Kernel &k : kAny) consider(k);
    return best->run(p, stream);
}

int product4(const char *who, Product4 &p, int64_t m, int64_t n, int64_t k, int experts, void *stream)
{
    if (!known(p.out)) return fail(OPEVO_E_ARG, "%s: unknown output type %d", who, p.out);
    if (m < 0 || n < 0 || m > (1 << 21) || n > (1 << 24)) return fail(OPEVO_E_ARG, "%s: %lld rows (at most 2^21) and %lld columns (at most 2^24)", who, (long long)m, (long long)n);
    if (k < 1 || k > (1 << 24)) return fail(OPEVO_E_ARG, "%s: K = %lld (1 to 2^24)", who, (long long)k);
    if (m == 0 || n == 0) return OPEVO_OK;
    const int64_t bytes = (k + 1) / 2, blocks = (k + 31) / 32;
    if (int rc = check_rows(who, "a", p.a, p.lda, bytes, 1)) return rc;
    if (int rc = check_rows(who, "scale_a", p.sa, p.ldsa, blocks, 1)) return rc;
    if (int rc = check_rows(who, "b", p.b, p.ldb, bytes, 1)) return rc;
    if (int rc = check_rows(who, "scale_b", p.sb, p.ldsb, blocks, 1)) return rc;
    if (int rc = check_rows(who, "c", p.c, p.ldc, n, size_of(p.out))) return rc;
    p.m = m; p.n = (int)n; p.k = (int)bytes; p.blocks = (int)blocks; p.odd = k % 2 != 0; p.experts = experts;
    return run_product4(p, static_cast<hipStream_t>(stream));
}

}  // namespace

extern "C" int opevo_matmul_mx4(const uint8_t *a, int64_t lda, const uint8_t *scale_a, int64_t ld_scale_a, const uint8_t *b, int64_t ldb, const uint8_t *scale_b,
                                int64_t ld_scale_b, void *c, int64_t ldc, int out_dtype, int64_t M, int64_t N, int64_t K, void *stream)
{
    Product4 p = {a, b, scale_a, scale_b, (long)lda, (long)ldb, (long)ld_scale_a, (long)ld_scale_b, nullptr, 0, c, (long)ldc, out_dtype, 0, 0, 0, 0, false};
    return product4("matmul_mx4", p, M, N, K, 0, stream);
}

extern "C" int opevo_matmul_mx4_grouped(const uint8_t *a, int64_t lda, const uint8_t *scale_a, int64_t ld_scale_a, const uint8_t *b, int64_t ldb, const uint8_t *scale_b,
                                        int64_t ld_scale_b, const int32_t *offsets, int experts, void *c, int64_t ldc, int out_dtype, int64_t rows, int64_t N, int64_t K,
                                        void *stream)
{
    const char *who = "matmul_mx4_grouped";
    if (experts < 1 || experts > OPEVO_ROUTE_MAX_EXPERTS) return fail(OPEVO_E_ARG, "%s: %d experts (1 to %d)", who, experts, OPEVO_ROUTE_MAX_EXPERTS);
    if (rows > 0 && N > 0 && (!offsets || reinterpret_cast<uintptr_t>(offsets) % 4)) return fail(OPEVO_E_ARG, "%s: offsets is NULL or not aligned to 4 bytes", who);
    Product4 p = {a, b, scale_a, scale_b, (long)lda, (long)ldb, (long)ld_scale_a, (long)ld_scale_b, offsets, experts, c, (long)ldc, out_dtype, 0, 0, 0, 0, false};
    return product4(who, p, rows, N, K, experts, stream);
}
