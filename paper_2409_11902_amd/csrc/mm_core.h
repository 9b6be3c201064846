// Matrix products C = A B^T by matrix instructions, with the work on C done where it lies in registers: the classifier's loss
// (loss.hip) and the orthogonalised update (muon.hip) are such products with different endings.
//
// A has M rows, B has N, and the sum runs over K.  Each operand comes in one of two layouts:
//   kAlong: K runs along a row of memory (row index m or n)
//   kDown : K is the row of memory (m or n runs along it); the transposing LDS read makes fragments of it
// and in one of these number formats:
//   Bf16  : bfloat16, one product
//   Split : a float as the sum of two half-precision numbers, x = hi + lo.  hi holds 11 bits of the significand and lo the next
//           12 (its sign is one of them): 2^-23 of x is lost.  hi hi + hi lo + lo hi leaves out lo lo, at most 2^-22 of a product and
//           2e-8 of it in the mean, so sums come out as float arithmetic has them, from three products at 16 times the
//           float instruction's rate.  A row of memory holds 8 hi, 8 lo, 8 hi, ...: a chunk of 16 bytes of one kind after one of
//           the other, so that both formats are staged alike, 128 bytes of K to a row and pass.  Numbers are stored times a
//           power of two that the caller takes out again: lo is subnormal of numbers below 2^-15 of those that are stored as 2^13 and more, and
//           they are off by up to 2^-25 as stored.
//
//   Raw   : floats as they lie, by the float instruction.  It needs no powers of two and no pass beforehand, and is what products of few
//           rows take, whose time is that of reading the other operand once.  A chunk holds 4 numbers, two of them the 8 that a
//           chunk of hi and one of lo hold.
//   Bf16Odd, RawOdd: the same of rows that start on 4 bytes and not on 16: 4 bytes to a lane and load in the place of 16.
//
// A workgroup of WM x WN waves owns a tile of C; a wave holds MI x NI accumulators of 32 x 32.  Tiles go from global memory straight
// into one of two LDS buffers while the other is multiplied, and a step's fragments are read while the step before is multiplied: the
// workgroup meets once a pass, after the last fragments of a buffer are in registers, with a step's products still to issue.  Lanes past
// a matrix's edge are given an offset past the descriptor's range and load zeros.
#pragma once
#include "train_ends.h"

namespace cac {
namespace mm {

typedef __attribute__((ext_vector_type(8))) _Float16 f16x8;
typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8;
typedef __attribute__((ext_vector_type(4))) short s16x4;
typedef __attribute__((ext_vector_type(8))) short s16x8;
typedef __attribute__((ext_vector_type(16))) float f32x16;
typedef __attribute__((ext_vector_type(4))) float f32x4;
typedef __attribute__((ext_vector_type(2))) uint32_t u32x2;
typedef __attribute__((ext_vector_type(4))) uint32_t u32x4;

enum class Lay { kAlong, kDown };
struct Bf16 { static constexpr int kParts = 1, kUnit = 16; static constexpr bool kRaw = false; }; // (kUnit: bytes to a lane and load)
struct Bf16Odd { static constexpr int kParts = 1, kUnit = 4; static constexpr bool kRaw = false; };
struct Split { static constexpr int kParts = 2, kUnit = 16; static constexpr bool kRaw = false; };
struct Raw { static constexpr int kParts = 2, kUnit = 16; static constexpr bool kRaw = true; };
struct RawOdd { static constexpr int kParts = 2, kUnit = 4; static constexpr bool kRaw = true; };
// units that n numbers of a row take: whole eights where rows are padded to them, else no more than there are
template <class P> __host__ __device__ constexpr int units(int n)
{
    return P::kRaw || P::kUnit == 4 ? (n * (P::kRaw ? 4 : 2) + P::kUnit - 1) / P::kUnit : P::kParts * ((n + 7) / 8);
}

constexpr uint32_t kNowhere = 0x80000000u; // an offset past every descriptor's range

// Rows of H that count: whose label is a class and not the one that is ignored.
struct Counts {
    const int64_t *labels; // null: every row counts
    int64_t ignore;
    int classes;
    __device__ __forceinline__ bool operator()(int row) const
    {
        if (!labels) return true;
        const int64_t l = labels[row];
        return l != ignore && l >= 0 && l < classes;
    }
};

struct Params {
    const void *a, *b;
    long lda, ldb;             // bytes from a row of memory to the next, below 2^23
    long a_batch, b_batch;     // bytes from a matrix to the next
    int M, N, K;
    const int *m_dev, *k_dev;  // where set: the rows (the terms) that there really are, at most M (K)
    int tiles_n, tiles;        // tiles in a row of them, and of one matrix: all, or those on and above the diagonal
    int batch, slices;         // matrices; parts that each sum is formed in
    int group;                 // tile rows that one XCD walks together
    int kt_slice;              // passes over K of one slice of the sum
    Counts counts_m;           // where an ending says so, rows of a that count: the others are zeros, whatever stands there
};

template <class P, int R> constexpr int kPass = R / 2 / P::kParts; // terms of the sum in one pass, R bytes of K to a row

// Which chunk of 16 bytes of a memory row stands where in LDS.  kAlong: rows of R bytes of which 16 are read together at one chunk; kDown: half a
// wave reads 4 rows together at 32 neighbouring columns (of every other chunk where a row has two parts).
template <class P, Lay L, int T, int R> __device__ __forceinline__ int swizzle(int row)
{
    static_assert(R == 128, "eight chunks to a row");
    if (L == Lay::kAlong) return (row >> 1) & 7;
    if (P::kParts == 2) return ((row & 1) << 3) ^ ((row >> 1) & 1);
    if (T == 64) return (row & 2) << 1;
    return (row & 3) << 2;
}

// 16 (4) bytes a lane from `offset` in `rs` to LDS, side by side from the uniform address `to` on.  Written out, because the compiler makes
// every transposing LDS read that follows one of its own wait for all of them; meet() says when they have arrived.  No register is
// written, so there is nothing that could be overwritten under way.
template <int UNIT> __device__ __forceinline__ void load_to_lds(u32x4 rs, uint32_t offset, uint32_t to)
{
    if (UNIT == 4) asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dword %1, %2, 0 offen lds" ::"s"(to), "v"(offset), "s"(rs) : "memory");
    else asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" ::"s"(to), "v"(offset), "s"(rs) : "memory"); // (m0 has no other use in these kernels)
}

// One operand's way into LDS: T rows of C by one pass of K, R T bytes, by NW waves.
template <class P, Lay L, int T, int R, int NW, bool COUNTS> struct Stage {
    static constexpr int kUnit = P::kUnit, kOf16 = 16 / kUnit;             // bytes to a lane and load; units in a chunk
    static constexpr int kLoads = T * R / (64 * kUnit) / NW;               // per wave and pass
    static constexpr int kRowBytes = L == Lay::kAlong ? R : T * 2 * P::kParts;
    static constexpr int kUnits = kRowBytes / kUnit, kStep = NW * 64 / kUnits; // units of a row; rows from a load to the next
    static_assert(kLoads * 64 * kUnit * NW == T * R && kStep * kUnits == NW * 64, "whole loads");
    const char *base; // of the pass to load next
    long step;        // bytes from a pass to the next
    uint32_t off[kLoads];
    int at;           // the lane's unit of a row in even loads (kAlong), its first row (kDown)
    int left;         // units (kAlong) or rows (kDown) of K from the pass to load next on

    // first: first row of C; count: rows of C in the matrix; K: terms; kt: first pass, kt1: behind the last
    __device__ __forceinline__ void init(const char *p, long ld, int first, int count, int K, int kt, int kt1, int wave, int lane, const Counts &counts)
    {
        const int row0 = (wave * 64 + lane) / kUnits, slot = (wave * 64 + lane) % kUnits;
        const int columns = units<P>(count) - units<P>(first); // kDown: units from the tile's first on
        if (L == Lay::kAlong) {
            static_assert(L != Lay::kAlong || kStep % 16 == 0 || kStep == 8, "a lane's unit is the same in every load, or every other");
            at = slot ^ swizzle<P, L, T, R>(row0) * kOf16;
            left = min(units<P>(K), kt1 * kUnits) - kt * kUnits;
            base = p + (long)first * ld + (long)kt * R;
            step = R;
        } else {
            at = row0;
            left = min(K, kt1 * kPass<P, R>) - kt * kPass<P, R>;
            base = p + (long)first * 2 * P::kParts + (long)kt * kPass<P, R> * ld;
            step = kPass<P, R> * ld;
        }
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            const int row = row0 + i * kStep, c = slot ^ swizzle<P, L, T, R>(row) * kOf16;
            bool there = L == Lay::kAlong ? first + row < count : c < columns;
            if (COUNTS && there) there = counts(first + row);
            off[i] = there ? (uint32_t)(row * (int)ld + c * kUnit) : kNowhere;
        }
    }
    // load i of the next pass into LDS at byte address `lds`; behind the last pass that is zeros
    __device__ __forceinline__ void load_one(int i, uint32_t lds, int wave)
    {
        const uint64_t from = (uint64_t)(uintptr_t)base;
        const u32x4 rs = {(uint32_t)from, (uint32_t)(from >> 32) & 0xffffu, 0x7fffffffu, 0x00020000u};
        const int here = L == Lay::kDown ? at + i * kStep : kStep == 8 && i % 2 ? at ^ 4 * kOf16 : at; // (8 rows on: four chunks apart)
        const uint32_t o = here < left ? off[i] : kNowhere;
        const uint32_t to = __builtin_amdgcn_readfirstlane(lds + (i * NW + wave) * 64 * kUnit);
        load_to_lds<kUnit>(rs, o, to);
    }
    __device__ __forceinline__ void advance()
    {
        base += step;
        left -= L == Lay::kAlong ? kUnits : kPass<P, R>;
    }
    __device__ __forceinline__ void load(uint32_t lds, int wave)
    {
#pragma unroll
        for (int i = 0; i < kLoads; ++i) load_one(i, lds, wave);
        advance();
    }
};

// Fragments of one operand: 32 rows of C by 16 terms, 8 terms to a lane (terms 8 * (lane / 32) on, row lane % 32).
template <class P, Lay L, int T, int R> struct Frag {
    static constexpr int kRowBytes = L == Lay::kAlong ? R : T * 2 * P::kParts;
    uint32_t at;  // the lane's place in the wave's first block
    uint32_t x;   // what a chunk's number is combined with
    int block0;   // the wave's first block of 32 rows of C

    __device__ __forceinline__ void init(int block, int lane)
    {
        block0 = block;
        if (L == Lay::kAlong) {
            at = (block * 32 + (lane & 31)) * R;
            x = swizzle<P, L, T, R>(lane & 31) ^ ((lane >> 5) * P::kParts);
        } else {
            const int row = 8 * (lane >> 5) + ((lane & 15) >> 2);
            at = row * kRowBytes + (lane & 1) * 8;
            x = swizzle<P, L, T, R>(row);
        }
    }
    // block blk of the wave, 16 terms from 16 s on, part 0 (hi, or the only one) or 1 (lo)
    __device__ __forceinline__ s16x8 get(uint32_t lds, int blk, int s, int part, int lane) const
    {
        typedef __attribute__((address_space(3))) s16x4 lds4;
        typedef __attribute__((address_space(3))) s16x8 lds8;
        if (L == Lay::kAlong) {
            const uint32_t c = x ^ (uint32_t)(s * 2 * P::kParts + part);
            return *(lds8 *)(uintptr_t)(lds + at + blk * 32 * R + (c << 4));
        }
        if constexpr (P::kRaw) { // four terms of a column, one below the other
            const uint32_t n = (block0 + blk) * 32 + (lane & 31);
            union { float f[4]; s16x8 v; } r;
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const int row = s * 16 + 8 * (lane >> 5) + part * 4 + k;
                r.f[k] = *(__attribute__((address_space(3))) float *)(uintptr_t)(lds + row * kRowBytes + (((n >> 2) ^ swizzle<P, L, T, R>(row)) << 4) + (n & 3) * 4);
            }
            return r.v;
        }
        const uint32_t col = (block0 + blk) * 4 + ((lane >> 4) & 1) * 2 + ((lane & 3) >> 1);
        const uint32_t c = (col * P::kParts + part) ^ x;
        const uint32_t p = lds + at + (c << 4) + s * 16 * kRowBytes;
        union { s16x4 h[2]; s16x8 v; } r;
        r.h[0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4 *)(uintptr_t)p);
        r.h[1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4 *)(uintptr_t)(p + 4 * kRowBytes));
        return r.v;
    }
};

template <class P> __device__ __forceinline__ f32x16 product(s16x8 a, s16x8 b, f32x16 c)
{
    union { s16x8 s; f16x8 h; bf16x8 b; } x, y;
    x.s = a;
    y.s = b;
    if (P::kParts == 2) return __builtin_amdgcn_mfma_f32_32x32x16_f16(x.h, y.h, c, 0, 0, 0);
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(x.b, y.b, c, 0, 0, 0);
}

__device__ __forceinline__ f32x4 as_floats(s16x8 v)
{
    union { s16x8 s; f32x4 f; } x;
    x.s = v;
    return x.f;
}

// What an ending may say about its product.
struct Ending { static constexpr bool kSymmetric = false, kCountsM = false, kGated = false, kOther = false; };
// (kGated: only tiles whose columns an ending's wanted() asks for; kOther: its operand_a() says where a tile's rows of a lie)

// ---- a float as two halves.  x is fixed first: left to itself the compiler takes hi from a product's rounded value and lo from the
// product, and where those lie on two sides of a half-precision number's middle, hi + lo is off by a unit of hi.
__device__ __forceinline__ void split_float(float x, _Float16 *hi, _Float16 *lo)
{
    asm("" : "+v"(x));
    *hi = (_Float16)x;
    *lo = (_Float16)(x - (float)*hi);
}
// four neighbours of a row (n a multiple of 4) to where a split matrix's row `row` holds them
__device__ __forceinline__ void store_split(char *row, int n, const float (&v)[4])
{
    union { _Float16 h[4]; u32x2 u; } hi, lo;
#pragma unroll
    for (int e = 0; e < 4; ++e) split_float(v[e], &hi.h[e], &lo.h[e]);
    char *c = row + (n >> 3) * 32 + (n & 4) * 2;
    *(u32x2 *)c = hi.u;
    *(u32x2 *)(c + 16) = lo.u;
}
__device__ __forceinline__ void load_split(const char *row, int n, float (&v)[4])
{
    union { _Float16 h[4]; u32x2 u; } hi, lo;
    const char *c = row + (n >> 3) * 32 + (n & 4) * 2;
    hi.u = *(const u32x2 *)c;
    lo.u = *(const u32x2 *)(c + 16);
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = (float)hi.h[e] + (float)lo.h[e];
}

// ---- Newton-Schulz products (muon.hip, muon_narrow.hip)
constexpr float kNsA = 3.4445f, kNsB = -4.7750f, kNsC = 2.0315f, kNsEps = 1e-7f;
constexpr float kNsStore = 4096.f, kNsTake = 1.f / 4096.f; // what X, A and the polynomial are stored times
// A matrix whose norm is little beside kNsEps starts, and a few steps at 3.4445 apiece later ends, with small numbers: its X is
// stored times 2^lift too, by as much as the last step leaves room for.
__device__ __forceinline__ int ns_lift(double norm, int steps)
{
    const double last = norm / (norm + (double)kNsEps) * pow((double)kNsA, (double)steps);
    if (!(last > 0.0 && last < 1.0)) return 0;
    return -ilogb(last) - 1;
}

// ---- 32 rows of a wave's part of C on their way to memory.  A lane holds four neighbours of a row, and a store of them touches 32 rows at
// 8 or 16 bytes each; through LDS they become stores of 16 bytes a lane, whole lines side by side.
enum class Fmt { kBf16, kF32, kSplit };
template <Fmt F, int NI> struct RowBlock {
    static constexpr int kRow = 32 * NI * (F == Fmt::kBf16 ? 2 : 4), kPitch = kRow + 16; // bytes
    static __device__ __forceinline__ void put(unsigned char *lds, int lane, int j, int q, const float (&v)[4])
    {
        unsigned char *r = lds + (lane & 31) * kPitch;
        const int n = j * 32 + q * 8 + (lane >> 5) * 4;
        if (F == Fmt::kSplit) {
            store_split((char *)r, n, v);
        } else if (F == Fmt::kF32) {
            *(f32x4 *)(r + n * 4) = f32x4{v[0], v[1], v[2], v[3]};
        } else {
            u32x2 u;
            u[0] = f32x2_to_bf16x2(v[0], v[1]);
            u[1] = f32x2_to_bf16x2(v[2], v[3]);
            *(u32x2 *)(r + n * 2) = u;
        }
    }
    // the mirror image of a block of 32 x 32, in rows of 32: a lane's four become four rows' (NI = 1)
    static __device__ __forceinline__ void put_mirrored(unsigned char *lds, int lane, int q, const float (&v)[4])
    {
        const int n = q * 8 + (lane >> 5) * 4, m = lane & 31;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            _Float16 hi, lo;
            split_float(v[e], &hi, &lo);
            unsigned char *c = lds + (n + e) * kPitch + (m >> 3) * 32 + (m & 7) * 2;
            *(_Float16 *)c = hi;
            *(_Float16 *)(c + 16) = lo;
        }
    }
    // store(row, byte offset in the row, 16 bytes) for all of it; the block's LDS is free afterwards
    template <class Fn> static __device__ __forceinline__ void each(unsigned char *lds, int lane, Fn store)
    {
        asm volatile("" ::: "memory"); // (a wave's LDS accesses are in order; other lanes' stores are read here)
        __builtin_amdgcn_wave_barrier();
        u32x4 v[kRow / 32];
#pragma unroll
        for (int c = 0; c < kRow / 32; ++c) {
            const int at = c * 64 + lane;
            v[c] = *(const u32x4 *)(lds + at / (kRow / 16) * kPitch + at % (kRow / 16) * 16);
        }
        asm volatile("" ::: "memory");
        __builtin_amdgcn_wave_barrier();
#pragma unroll
        for (int c = 0; c < kRow / 32; ++c) {
            const int at = c * 64 + lane;
            store(at / (kRow / 16), at % (kRow / 16) * 16, v[c]);
        }
    }
};

// Where a wave's part of C lies.  acc[mi][ni][4 q + e] is C[m][n] of m = m0 + 32 mi + lane % 32 and
// n = n0 + 32 ni + 8 q + 4 (lane / 32) + e: a lane holds four neighbours of a row of C.
struct Place {
    int m0, n0;         // the wave's first row and column
    int M, N;           // extents, M as it really is
    int batch, slice;
    int tm, tn;         // the tile
    int part;           // the wave's place among the waves that share a row of C
    unsigned char *lds; // the wave's own, free at the end
    int lds_rows;       // from there to that of the wave with the rows that follow
    int lane;
};

// How a workgroup's tile is made of waves' parts, and how it is staged: R bytes of K to a row and pass, ST passes in LDS.
// MIXED: a pass' loads are issued one between two products (a wave waits to issue a load while others' are taken in, 16 cycles each, and
// issues nothing else meanwhile), else all together.
template <int WM_, int WN_, int MI_, int NI_, int R_, int ST_, int PER_CU, bool MIXED = false> struct Shape {
    static constexpr bool kMixed = MIXED;
    static constexpr int WM = WM_, WN = WN_, MI = MI_, NI = NI_, R = R_, ST = ST_, kWaves = WM * WN, kThreads = 64 * kWaves;
    static constexpr int TM = 32 * MI * WM, TN = 32 * NI * WN, kBuffer = (TM + TN) * R, kLds = ST * kBuffer;
    static constexpr int kPerSimd = PER_CU * kWaves / 4; // waves that registers are shared by
};
// Measured, with what bounds them (a library's product of 8192 cubed reaches 1.23 PFLOP/s in bfloat16 and 1.33 in half precision on the same
// card, 1.33 / 3 = 0.44 for three of them; bare matrix instructions 1.7).  Under the two largest tiles the clock falls to 1.8 to 2.0 GHz of 2.4, and
// matrix instructions are on 54 to 60 % of its cycles where sums are long (38 % of 1024 terms); LDS bank conflicts take 2 % at most under any:
typedef Shape<2, 4, 4, 2, 128, 2, 1> Big;    // 256 x 256: the clock.  7373 x 131072 x 4096 bfloat16 1.07 PFLOP/s; 4096 cubed Split 0.36
typedef Shape<2, 6, 3, 1, 128, 3, 1> Wide;   // 192 x 192: as Big, where its tiles fill the compute units better.  4096 cubed, symmetric, Split 0.31
typedef Shape<2, 4, 2, 1, 128, 2, 2> Middle; // 128 x 128: what a compute unit takes in, 35 to 50 KB a us.  512 x 4608 x 512, three of them, Split 0.25
typedef Shape<2, 2, 1, 1, 128, 3, 3> Small;  // 64 x 64: latency (matrix instructions on 3 to 20 % of cycles).  A pass takes 0.27 us alone and 0.2 to 0.3 with two others beside it
typedef Shape<1, 4, 1, 1, 128, 3, 2> Low;    // 32 x 128, for few rows of floats: reading b.  16 x 100000 x 1024 3.0 to 3.7 TB/s

// All but the N youngest loads have arrived, the fragments asked for are in registers, and every wave of the workgroup says so.
template <int N> __device__ __forceinline__ void meet()
{
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(N) : "memory");
}

// One workgroup's tile, as workgroup `block` of the product.
template <class P, Lay LA, Lay LB, class S, class Epi>
__device__ __forceinline__ void mm_tile(const Params &p, const typename Epi::Params &e, int block, unsigned char *smem)
{
    constexpr int MI = S::MI, NI = S::NI, TM = S::TM, TN = S::TN;
    constexpr int kSteps = S::R / 32 / P::kParts; // of 16 terms, in a pass
    static_assert(kSteps % 2 == 0, "a pass ends with the fragments' registers that it began with");
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int M = p.m_dev ? min(p.M, *p.m_dev) : p.M, K = p.k_dev ? min(p.K, *p.k_dev) : p.K;

    // Workgroups go round the eight XCDs, each with an L2 of its own: an XCD gets a run of neighbouring tiles of the rows that there
    // really are, slice after slice (a slice's tiles share its terms and no other's), and walks it in groups of `group` tile rows.
    const int tiles_m = (M + TM - 1) / TM, tiles = Epi::kSymmetric ? p.tiles : tiles_m * p.tiles_n, all = tiles * p.slices * p.batch;
    const int per = (all + 7) / 8, t = (block & 7) * per + (block >> 3);
    if ((block >> 3) >= per || t >= all) return;
    // (said to be uniform, which quotients of uniform numbers are not seen to be)
    const int batch = __builtin_amdgcn_readfirstlane(t / (tiles * p.slices));
    const int slice = __builtin_amdgcn_readfirstlane(t / tiles) - batch * p.slices, tt = t - (batch * p.slices + slice) * tiles;
    int tm, tn;
    if (Epi::kSymmetric) { // the tiles on and above the diagonal, row by row: row i has tiles_m - i
        tm = __builtin_amdgcn_readfirstlane((int)(tiles_m + 0.5f - sqrtf((tiles_m + 0.5f) * (tiles_m + 0.5f) - 2.f * tt)));
        while (tm > 0 && tm * tiles_m - tm * (tm - 1) / 2 > tt) --tm;
        while ((tm + 1) * tiles_m - (tm + 1) * tm / 2 <= tt) ++tm;
        tn = tt - (tm * tiles_m - tm * (tm - 1) / 2) + tm;
    } else {
        const int g0 = __builtin_amdgcn_readfirstlane(tt / (p.group * p.tiles_n)) * p.group, gr = min(p.group, tiles_m - g0), gi = tt - g0 * p.tiles_n;
        tn = __builtin_amdgcn_readfirstlane(gi / gr);
        tm = g0 + gi - tn * gr;
    }

    if constexpr (Epi::kGated)
        if (!Epi::wanted(e, tn * TN, min(p.N - tn * TN, TN), lane)) return;
    const void *from_a = p.a;
    if constexpr (Epi::kOther) from_a = Epi::operand_a(e, p.a, tm * TM, min(M - tm * TM, TM), lane);

    const int passes = (K + kPass<P, S::R> - 1) / kPass<P, S::R>;
    const int kt0 = slice * p.kt_slice, kt1 = min(passes, kt0 + p.kt_slice);

    f32x16 acc[MI][NI];
#pragma unroll
    for (int i = 0; i < MI; ++i)
#pragma unroll
        for (int j = 0; j < NI; ++j)
#pragma unroll
            for (int r = 0; r < 16; ++r) acc[i][j][r] = 0.f;

    Stage<P, LA, TM, S::R, S::kWaves, Epi::kCountsM> sa;
    Stage<P, LB, TN, S::R, S::kWaves, false> sb;
    sa.init((const char *)from_a + batch * p.a_batch, p.lda, tm * TM, M, K, kt0, kt1, wave, lane, p.counts_m);
    sb.init((const char *)p.b + batch * p.b_batch, p.ldb, tn * TN, p.N, K, kt0, kt1, wave, lane, p.counts_m);
    const int wm = wave / S::WN, wn = wave % S::WN;
    Frag<P, LA, TM, S::R> fa;
    Frag<P, LB, TN, S::R> fb;
    fa.init(wm * MI, lane);
    fb.init(wn * NI, lane);
    const uint32_t lds = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) unsigned char *)smem;
    const uint32_t lds_end = lds + S::kLds;

    auto load = [&](uint32_t to) {
        sa.load(to, wave);
        sb.load(to + TM * S::R, wave);
    };
    s16x8 a[2][P::kParts][MI], b[2][P::kParts][NI];
    auto read = [&](int r, uint32_t from, int s) {
#pragma unroll
        for (int h = 0; h < P::kParts; ++h) {
#pragma unroll
            for (int i = 0; i < MI; ++i) a[r][h][i] = fa.get(from, i, s, h, lane);
#pragma unroll
            for (int j = 0; j < NI; ++j) b[r][h][j] = fb.get(from + TM * S::R, j, s, h, lane);
        }
    };
    constexpr int kAhead = (S::ST - 2) * (decltype(sa)::kLoads + decltype(sb)::kLoads); // loads younger than the next pass's
    if (kt0 < kt1) {
        uint32_t cur = lds;
#pragma unroll
        for (int i = 0; i < S::ST - 1; ++i) load(lds + i * S::kBuffer);
        meet<kAhead>();
        load(lds_end - S::kBuffer);
        read(0, lds, 0);
        for (int kt = kt0; kt < kt1; ++kt) {
#pragma unroll
            for (int s = 0; s < kSteps; ++s) {
                if (s + 1 < kSteps) {
                    read((s + 1) & 1, cur, s + 1);
                } else {
                    const uint32_t next = cur + S::kBuffer == lds_end ? lds : cur + S::kBuffer;
                    meet<kAhead>(); // the next pass has arrived; this one's last fragments are in registers
                    if (!S::kMixed) load(cur);
                    read((s + 1) & 1, next, 0);
                    if constexpr (S::kMixed) {
                        static_assert(!S::kMixed || (!P::kRaw && P::kParts == 1), "bfloat16");
                        constexpr int kA = decltype(sa)::kLoads, kB = decltype(sb)::kLoads;
                        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                        for (int k = 0; k < MI * NI; ++k) {
                            acc[k / NI][k % NI] = product<P>(b[s & 1][0][k % NI], a[s & 1][0][k / NI], acc[k / NI][k % NI]);
                            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                            for (int i = k * (kA + kB) / (MI * NI); i < (k + 1) * (kA + kB) / (MI * NI); ++i) {
                                if (i < kA) sa.load_one(i, cur, wave);
                                else sb.load_one(i - kA, cur + TM * S::R, wave);
                            }
                            __builtin_amdgcn_sched_barrier(0);
                        }
                        sa.advance();
                        sb.advance();
                    }
                    cur = next;
                }
                if (S::kMixed && s + 1 == kSteps) continue;
                __builtin_amdgcn_sched_barrier(0);
                if constexpr (P::kRaw) { // (term e of a lane's eight: one of the first 8 with one of the second)
#pragma unroll
                    for (int h = 0; h < 2; ++h)
#pragma unroll
                        for (int e = 0; e < 4; ++e)
#pragma unroll
                            for (int i = 0; i < MI; ++i)
#pragma unroll
                                for (int j = 0; j < NI; ++j)
                                    acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x2f32(as_floats(b[s & 1][h][j])[e], as_floats(a[s & 1][h][i])[e], acc[i][j], 0, 0, 0);
                } else {
#pragma unroll
                        for (int h = 0; h < 2 * P::kParts - 1; ++h) // hi hi, then hi lo and lo hi
#pragma unroll
                        for (int i = 0; i < MI; ++i)
#pragma unroll
                            for (int j = 0; j < NI; ++j) acc[i][j] = product<P>(b[s & 1][h & 1][j], a[s & 1][h >> 1][i], acc[i][j]);
                }
                __builtin_amdgcn_sched_barrier(0);
            }
        }
        meet<0>(); // nothing is on its way into LDS when the workgroup ends
    }
    Place at;
    at.m0 = tm * TM + wm * 32 * MI;
    at.n0 = tn * TN + wn * 32 * NI;
    at.M = M;
    at.N = p.N;
    at.batch = batch;
    at.slice = slice;
    at.tm = tm;
    at.tn = tn;
    at.part = tn * S::WN + wn;
    at.lane = lane;
    at.lds = smem + wave * (S::kLds / S::kWaves / 16 * 16);
    at.lds_rows = S::WN * (S::kLds / S::kWaves / 16 * 16);
    Epi::template run<MI, NI>(e, acc, at);
}

template <class P, Lay LA, Lay LB, class S, class Epi>
__global__ void __launch_bounds__(S::kThreads, S::kPerSimd) mm_kernel(const Params p, const typename Epi::Params e)
{
    extern __shared__ __align__(1024) unsigned char smem[];
    mm_tile<P, LA, LB, S, Epi>(p, e, blockIdx.x, smem);
}

// ---- host
inline int cdiv(long a, long b) { return (int)((a + b - 1) / b); }

// Which tile a product takes, and in how many slices its sum is formed.
enum { kSmall, kMiddle, kWide, kBig, kLow, kShapes };
enum Format { kBf16, kSplit, kRaw };
typedef TileChoice Choice;
constexpr int kRows[kShapes] = {64, 128, 192, 256, 32}, kColumns[kShapes] = {64, 128, 192, 256, 128}; // of a tile
constexpr int kWaveColumns[kShapes] = {Small::WN, Middle::WN, Wide::WN, Big::WN, Low::WN};            // waves that a tile's columns fall to
constexpr int kTerms[] = {64, 32, 32};                                                                // of the sum, in a pass

// Microseconds of a product, from what a pass measured: on a compute unit with one workgroup, and with as many as it holds.
inline double product_us(int shape, Format f, long tiles, int passes, int slices)
{
    static const int kHolds[kShapes] = {3, 2, 1, 1, 2};
    static const double kAlone[kShapes][3] = {{0.27, 0.27, 0.5}, {0.77, 0.80}, {0, 1.75}, {1.95, 2.85}, {0, 0, 0.5}}, // (0: no such kernel)
                        kFull[kShapes][3] = {{0.62, 0.95, 1.4}, {1.12, 1.5}, {0, 1.75}, {1.95, 2.85}, {0, 0, 1.0}},
                        kOnce[kShapes] = {2.5, 3.5, 5.0, 6.0, 2.5};
    const long wgs = tiles * slices, round = 256L * kHolds[shape];
    const double n = cdiv(passes, slices), rest = (double)(wgs % round);
    double us = (wgs / round) * (kFull[shape][f] * n + kOnce[shape]);
    if (rest > 0) {
        const double share = rest <= 256 ? 0.0 : (rest - 256) / (round - 256);
        us += (kAlone[shape][f] + share * (kFull[shape][f] - kAlone[shape][f])) * n + kOnce[shape];
    }
    return us;
}
// A launch has fewer than 2^32 threads, its workgroups rounded up to the XCDs.
inline bool fits_grid(int shape, long workgroups)
{
    static const int kThreads[kShapes] = {Small::kThreads, Middle::kThreads, Wide::kThreads, Big::kThreads, Low::kThreads};
    return (workgroups + 7) / 8 * 8 * kThreads[shape] < 1L << 32;
}
inline long tiles_of(int shape, long M, long N, bool symmetric)
{
    const long m = cdiv(M, kRows[shape]), n = cdiv(N, kColumns[shape]);
    return symmetric ? m * (m + 1) / 2 : m * n;
}
// The cheapest of them; more than one slice costs the writing and reading of that many sums of 32 bits, and a launch.  (Over 150 products of 16
// to 6000 rows, columns and terms the one that this takes is 0.7 % (Split; Bf16 1.1 %) slower in the mean than the fastest of the four.)
inline Choice choose(Format f, long M, long N, int batch, long K, bool symmetric, int max_slices, bool small_only = false)
{
    Choice best{kSmall, 1};
    double least = 1e30;
    for (int shape = 0; shape < kShapes; ++shape) {
        if (small_only && shape != kSmall && shape != kLow) continue;
        if (shape == kWide && f != kSplit) continue; // (192 columns of bfloat16 are no whole number of swizzled chunks)
        if ((shape == kLow) != (f == kRaw && M <= kRows[kLow])) continue;
        if (f == kRaw && shape != kSmall && shape != kLow) continue; // (there are no others)
        const long tiles = tiles_of(shape, M, N, symmetric) * batch;
        const int passes = cdiv(K, kTerms[f]);
        for (int slices = 1; slices <= max_slices; slices += slices < 4 ? 1 : slices / 4 * 2) {
            if (slices > 1 && passes / slices < 4) break;
            if (slices > 1 && tiles * slices > 2048) break;
            if (!fits_grid(shape, tiles)) break; // (where none does the caller has to do with less at a time)
            double us = product_us(shape, f, tiles, passes, slices);
            if (slices > 1) us += 4.0 + 8e-6 / 2.5 * slices * tiles * kRows[shape] * kColumns[shape];
            if (us < least) {
                least = us;
                best = Choice{shape, slices};
            }
        }
    }
    return best;
}
// parts that a row's columns fall into, one to a wave
inline long wave_columns(long N, int shape) { return (long)cdiv(N, kColumns[shape]) * kWaveColumns[shape]; }

// Fills in the tiles; returns the workgroups (a multiple of the XCDs).
template <class S> inline unsigned place_tiles(Params *p, bool symmetric, int slices, int pass)
{
    const int tiles_m = cdiv(p->M, S::TM);
    p->tiles_n = cdiv(p->N, S::TN);
    p->tiles = symmetric ? tiles_m * (tiles_m + 1) / 2 : tiles_m * p->tiles_n;
    p->group = 8;
    p->slices = slices;
    p->kt_slice = cdiv(cdiv(p->K, pass), slices);
    return (unsigned)(8 * (((long)p->tiles * p->batch * slices + 7) / 8));
}
template <class P, Lay LA, Lay LB, class S, class Epi>
hipError_t launch_shape(Params p, const typename Epi::Params &e, int slices, hipStream_t st)
{
    static const hipError_t attr = hipFuncSetAttribute(reinterpret_cast<const void *>(mm_kernel<P, LA, LB, S, Epi>),
                                                       hipFuncAttributeMaxDynamicSharedMemorySize, S::kLds);
    if (attr != hipSuccess) return attr;
    const unsigned blocks = place_tiles<S>(&p, Epi::kSymmetric, slices, kPass<P, S::R>);
    hipLaunchKernelGGL((mm_kernel<P, LA, LB, S, Epi>), dim3(blocks), dim3(S::kThreads), S::kLds, st, p, e);
    return hipGetLastError();
}

template <class P, Lay LA, Lay LB, class Epi>
hipError_t launch(const Params &p, const typename Epi::Params &e, Choice c, hipStream_t st)
{
    if constexpr (P::kRaw) { // (the only ones that are asked for)
        if (c.shape == kLow) return launch_shape<P, LA, LB, Low, Epi>(p, e, c.slices, st);
        return launch_shape<P, LA, LB, Small, Epi>(p, e, c.slices, st);
    } else if constexpr (P::kUnit == 4) {
        return launch_shape<P, LA, LB, Small, Epi>(p, e, c.slices, st);
    } else {
        if (c.shape == kBig) return launch_shape<P, LA, LB, Big, Epi>(p, e, c.slices, st);
        if constexpr (P::kParts == 2)
            if (c.shape == kWide) return launch_shape<P, LA, LB, Wide, Epi>(p, e, c.slices, st);
        if (c.shape == kMiddle) return launch_shape<P, LA, LB, Middle, Epi>(p, e, c.slices, st);
        return launch_shape<P, LA, LB, Small, Epi>(p, e, c.slices, st);
    }
}

} // namespace mm
} // namespace cac
