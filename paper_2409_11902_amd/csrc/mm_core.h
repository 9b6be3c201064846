// Matrix products C = A B^T by matrix instructions, with the work on C done where it lies in registers: the classifier's loss
// (loss.hip) and the orthogonalised update (muon.hip) are such products with different endings.
//
// A has M rows, B has N, and the sum runs over K.  Each operand comes in one of two layouts:
//   kAlong: K runs along a row of memory (row index m or n)
//   kDown : K is the row of memory (m or n runs along it); the transposing LDS read makes fragments of it
// and in one of two number formats:
//   Bf16  : bfloat16, one product
//   Split : a float as the sum of two half-precision numbers, x = hi + lo.  hi holds 11 bits of the significand and lo the next
//           12 (its sign is one of them): 2^-23 of x is lost.  hi hi + hi lo + lo hi leaves out lo lo, at most 2^-22 of a product and
//           2e-8 of it in the mean, so sums come out as float arithmetic has them, from three products at 16 times the
//           float instruction's rate.  A row of memory holds 8 hi, 8 lo, 8 hi, ...: a chunk of 16 bytes of one kind after one of
//           the other, so that both formats are staged alike, 128 bytes of K to a row and pass.  Numbers are stored times a
//           power of two that the caller takes out again, which keeps lo out of the subnormal range.
//
// A workgroup of four waves (2 x 2) owns a tile of 64 I x 64 I; a wave holds I x I accumulators of 32 x 32.  Tiles go from global memory
// straight into one of two LDS buffers while the other is multiplied.  Lanes past a matrix's edge are given an offset past the
// descriptor's range and load zeros.
#pragma once
#include "common.h"

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
struct Bf16 { static constexpr int kParts = 1; };
struct Split { static constexpr int kParts = 2; };

constexpr uint32_t kNowhere = 0x80000000u; // an offset past every descriptor's range

struct Params {
    const void *a, *b;
    long lda, ldb;             // bytes from a row of memory to the next, below 2^23
    long a_batch, b_batch;     // bytes from a matrix to the next
    int M, N, K;
    const int *m_dev, *k_dev;  // where set: the rows (the terms) that there really are, at most M (K)
    int tiles_m, tiles_n, batch;
    int group;                 // tile rows that one XCD walks together
    int kt_slice;              // passes over K of one slice of the sum (blockIdx.y)
};

template <class P> constexpr int kPass = 64 / P::kParts; // terms of the sum in one pass

// Which chunk of 16 bytes of a memory row stands where in LDS.  kAlong: 128-byte rows of which 32 are read at one chunk; kDown: 8
// rows (0-3 and 8-11 of 16) are read together at 16 neighbouring columns.
template <class P, Lay L, int T> __device__ __forceinline__ int swizzle(int row)
{
    if (L == Lay::kAlong) return (row >> 1) & 7;
    if (P::kParts == 2) return ((row & 3) << 2) ^ ((row >> 3) & 1);
    if (T == 64) return (((row >> 1) & 1) | ((row >> 2) & 2)) << 1;
    return ((row & 3) | ((row >> 1) & 4)) << 1;
}

// One operand's way into LDS: T rows of C (T = 64 I) by one pass of K, 128 T bytes.
template <class P, Lay L, int T> struct Stage {
    static constexpr int kLoads = T / 32;                                  // per wave and pass, 1 KiB each
    static constexpr int kRowBytes = L == Lay::kAlong ? 128 : T * 2 * P::kParts;
    static constexpr int kChunks = kRowBytes / 16;
    const char *base;
    long step;     // bytes from a pass to the next
    uint32_t off[kLoads];
    int row0, chunk, left_total;
    long ld;

    // first: first row of C; count: rows of C in the matrix; K: terms
    __device__ __forceinline__ void init(const char *p, long ld_, int first, int count, int K, int kt0, int wave, int lane)
    {
        ld = ld_;
        if (L == Lay::kAlong) {
            chunk = (lane & 7) ^ (((wave & 1) << 2) + (lane >> 4));
            row0 = 0;
            left_total = P::kParts * ((K + 7) / 8); // chunks of a row
            base = p + (long)first * ld + (long)kt0 * 128;
            step = 128;
#pragma unroll
            for (int i = 0; i < kLoads; ++i) {
                const int row = (i * 4 + wave) * 8 + (lane >> 3);
                off[i] = first + row < count ? (uint32_t)(row * (int)ld + chunk * 16) : kNowhere;
            }
        } else {
            left_total = K; // rows of memory
            base = p + (long)first * 2 * P::kParts + (long)kt0 * kPass<P> * ld;
            step = kPass<P> * ld;
            row0 = (wave * 64 + lane) / kChunks;
            const int columns = P::kParts * ((count + 7) / 8) - first / 8 * P::kParts; // chunks from the tile's first on
#pragma unroll
            for (int i = 0; i < kLoads; ++i) {
                const int row = row0 + i * (256 / kChunks);
                const int c = ((wave * 64 + lane) % kChunks) ^ swizzle<P, L, T>(row);
                off[i] = c < columns ? (uint32_t)(row * (int)ld + c * 16) : kNowhere;
            }
            chunk = 0;
        }
    }
    // pass kt into LDS at byte address `lds`
    __device__ __forceinline__ void load(int kt, int kt0, uint32_t lds, int wave)
    {
        const rsrc_t rs = __builtin_amdgcn_make_buffer_rsrc(const_cast<char *>(base + (long)(kt - kt0) * step), 0, 0x7fffffff, 0x00020000);
        const int left = L == Lay::kAlong ? left_total - kt * 8 : left_total - kt * kPass<P>;
        const bool whole = left >= (L == Lay::kAlong ? 8 : kPass<P>);
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            uint32_t o = off[i];
            if (!whole) {
                const int at = L == Lay::kAlong ? chunk : row0 + i * (256 / kChunks);
                if (at >= left) o = kNowhere;
            }
            const uint32_t to = __builtin_amdgcn_readfirstlane(lds + (i * 4 + wave) * 1024);
            __builtin_amdgcn_raw_ptr_buffer_load_lds(rs, (__attribute__((address_space(3))) void *)(uintptr_t)to, 16, o, 0, 0, 0);
        }
    }
};

// Fragments of one operand: 32 rows of C by 16 terms, 8 terms to a lane (terms 8 * (lane / 32) on, row lane % 32).
template <class P, Lay L, int T> struct Frag {
    static constexpr int kRowBytes = Stage<P, L, T>::kRowBytes;
    uint32_t at;  // the lane's place in block 0
    uint32_t x;   // what a chunk's number is combined with
    int block0;   // the wave's first block of 32 rows of C

    __device__ __forceinline__ void init(int block, int lane)
    {
        block0 = block;
        if (L == Lay::kAlong) {
            at = (block * 32 + (lane & 31)) * 128;
            x = ((lane >> 1) & 7) ^ ((lane >> 5) * P::kParts);
        } else {
            const int row = 8 * (lane >> 5) + ((lane & 15) >> 2);
            at = row * kRowBytes + (lane & 1) * 8;
            x = swizzle<P, L, T>(row);
        }
    }
    // block blk of the wave, 16 terms from 16 s on, part 0 (hi, or the only one) or 1 (lo)
    __device__ __forceinline__ s16x8 get(uint32_t lds, int blk, int s, int part, int lane) const
    {
        typedef __attribute__((address_space(3))) s16x4 lds4;
        typedef __attribute__((address_space(3))) s16x8 lds8;
        if (L == Lay::kAlong) {
            const uint32_t c = x ^ (uint32_t)(s * 2 * P::kParts + part);
            return *(lds8 *)(uintptr_t)(lds + at + blk * 4096 + (c << 4));
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

// Where a wave's part of C lies.  acc[mi][ni][4 q + e] is C[m][n] of m = m0 + 32 mi + lane % 32 and
// n = n0 + 32 ni + 8 q + 4 (lane / 32) + e: a lane holds four neighbours of a row of C.
struct Place {
    int m0, n0;         // the wave's first row and column
    int M, N;           // extents, M as it really is
    int batch, slice;
    int tn, wn;         // the tile's column, the wave's column in it
    int lane;
};

template <class P, Lay LA, Lay LB, int I, class Epi>
__global__ void __launch_bounds__(256, I == 4 ? 1 : 2) mm_kernel(const Params p, const typename Epi::Params e)
{
    extern __shared__ __align__(1024) unsigned char smem[];
    constexpr int T = 64 * I, kTile = T * 128;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int M = p.m_dev ? min(p.M, *p.m_dev) : p.M, K = p.k_dev ? min(p.K, *p.k_dev) : p.K;

    // Workgroups go round the eight XCDs: each XCD gets a run of neighbouring tiles, and walks it in groups of `group` tile rows.
    const int tiles = p.tiles_m * p.tiles_n;
    const int per = (tiles * p.batch + 7) / 8;
    const int t = (blockIdx.x & 7) * per + (blockIdx.x >> 3);
    if ((int)(blockIdx.x >> 3) >= per || t >= tiles * p.batch) return;
    const int batch = t / tiles, tt = t - batch * tiles;
    const int g0 = tt / (p.group * p.tiles_n) * p.group, gr = min(p.group, p.tiles_m - g0), gi = tt - g0 * p.tiles_n;
    const int tm = g0 + gi % gr, tn = gi / gr;
    if (tm * T >= M) return;
    if (Epi::kSymmetric && tn < tm) return;

    const int passes = (K + kPass<P> - 1) / kPass<P>;
    const int kt0 = blockIdx.y * p.kt_slice, kt1 = min(passes, kt0 + p.kt_slice);

    f32x16 acc[I][I];
#pragma unroll
    for (int i = 0; i < I; ++i)
#pragma unroll
        for (int j = 0; j < I; ++j)
#pragma unroll
            for (int r = 0; r < 16; ++r) acc[i][j][r] = 0.f;

    Stage<P, LA, T> sa;
    Stage<P, LB, T> sb;
    sa.init((const char *)p.a + batch * p.a_batch, p.lda, tm * T, M, K, kt0, wave, lane);
    sb.init((const char *)p.b + batch * p.b_batch, p.ldb, tn * T, p.N, K, kt0, wave, lane);
    Frag<P, LA, T> fa;
    Frag<P, LB, T> fb;
    fa.init((wave >> 1) * I, lane);
    fb.init((wave & 1) * I, lane);
    const uint32_t lds = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) unsigned char *)smem;

    if (kt0 < kt1) {
        sa.load(kt0, kt0, lds, wave);
        sb.load(kt0, kt0, lds + kTile, wave);
    }
    for (int kt = kt0; kt < kt1; ++kt) {
        const uint32_t cur = lds + ((kt - kt0) & 1) * 2 * kTile, nxt = lds + ((kt - kt0 + 1) & 1) * 2 * kTile;
        __syncthreads();
        if (kt + 1 < kt1) {
            sa.load(kt + 1, kt0, nxt, wave);
            sb.load(kt + 1, kt0, nxt + kTile, wave);
        }
#pragma unroll
        for (int s = 0; s < 4 / P::kParts; ++s) {
            s16x8 a[P::kParts][I], b[P::kParts][I];
#pragma unroll
            for (int h = 0; h < P::kParts; ++h)
#pragma unroll
                for (int i = 0; i < I; ++i) {
                    a[h][i] = fa.get(cur, i, s, h, lane);
                    b[h][i] = fb.get(cur + kTile, i, s, h, lane);
                }
#pragma unroll
            for (int i = 0; i < I; ++i)
#pragma unroll
                for (int j = 0; j < I; ++j) {
                    acc[i][j] = product<P>(b[0][j], a[0][i], acc[i][j]);
                    if (P::kParts == 2) {
                        acc[i][j] = product<P>(b[P::kParts - 1][j], a[0][i], acc[i][j]);
                        acc[i][j] = product<P>(b[0][j], a[P::kParts - 1][i], acc[i][j]);
                    }
                }
        }
    }
    Place at;
    at.m0 = tm * T + (wave >> 1) * 32 * I;
    at.n0 = tn * T + (wave & 1) * 32 * I;
    at.M = M;
    at.N = p.N;
    at.batch = batch;
    at.slice = blockIdx.y;
    at.tn = tn;
    at.wn = wave & 1;
    at.lane = lane;
    Epi::template run<I>(e, acc, at);
}

// ---- host
inline int cdiv(long a, long b) { return (int)((a + b - 1) / b); }

// The tile's edge for a product of this size, in units of 64.
inline int choose_tile(long M, long N, int batch, int slices)
{
    for (int i : {4, 2}) {
        const long tiles = (long)cdiv(M, 64 * i) * cdiv(N, 64 * i) * batch * slices;
        if (tiles >= 256) return i;
    }
    return 1;
}

template <class P, Lay LA, Lay LB, class Epi, int I>
hipError_t launch_tile(Params p, const typename Epi::Params &e, int slices, hipStream_t st)
{
    constexpr int lds = 4 * 64 * I * 128;
    static const hipError_t attr =
        hipFuncSetAttribute(reinterpret_cast<const void *>(mm_kernel<P, LA, LB, I, Epi>), hipFuncAttributeMaxDynamicSharedMemorySize, lds);
    if (attr != hipSuccess) return attr;
    p.tiles_m = cdiv(p.M, 64 * I);
    p.tiles_n = cdiv(p.N, 64 * I);
    p.group = 8;
    p.kt_slice = cdiv(cdiv(p.K, kPass<P>), slices);
    const long total = (long)p.tiles_m * p.tiles_n * p.batch;
    hipLaunchKernelGGL((mm_kernel<P, LA, LB, I, Epi>), dim3((unsigned)(8 * ((total + 7) / 8)), slices), dim3(256), lds, st, p, e);
    return hipGetLastError();
}

template <class P, Lay LA, Lay LB, class Epi>
hipError_t launch(const Params &p, const typename Epi::Params &e, int tile, int slices, hipStream_t st)
{
    if (tile == 4) return launch_tile<P, LA, LB, Epi, 4>(p, e, slices, st);
    if (tile == 2) return launch_tile<P, LA, LB, Epi, 2>(p, e, slices, st);
    return launch_tile<P, LA, LB, Epi, 1>(p, e, slices, st);
}

// ---- a float as two halves
__device__ __forceinline__ void split_float(float x, _Float16 *hi, _Float16 *lo)
{
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

} // namespace mm
} // namespace cac
