// The orthogonalised update (muon.hip) of matrices whose shorter side is at most 64: what takes time there is launches, not products.
//
// A workgroup owns 64, 128 or 256 columns of its matrix (rows and columns are the shorter and the longer side here) as two halves in
// LDS, and the square products of 64 x 64 are cheap enough for every workgroup to form the polynomial by itself.  A matrix that one
// workgroup holds is done in one launch; a longer one takes a launch a step, which adds up the workgroups' parts of X X^T, forms the
// polynomial, multiplies its columns by it and leaves its part of the next X X^T.  No launch is spent on the norm: it is the
// trace of U U^T, and a workgroup's columns of U are stored times a power of two of their own until it is known.
// 64 x 64 takes 17 us, all of it one workgroup's chain of five steps of 3 us, each three products that wait for the one before;
// four of 64 x 576 take 53 us, in six launches of 9.
#include "mm_core.h"

namespace cac {

namespace {

using namespace mm;

constexpr float kA = kNsA, kB = kNsB, kC = kNsC, kTake = kNsTake, kStore = kNsStore;
constexpr int kSide = 64, kSquare = kSide * 256;       // bytes of a square matrix in LDS
// The power of two of columns that hold zeros alone, above every other's (which are 12 + 148 at most): the smallest is what all slices are brought to.
constexpr int kNone = 256;

struct Args {
    const void *G;
    float *M;
    void *out;
    int r, n;          // shorter, longer side
    int tall;          // element (i, j) lies at [j][i]
    int nesterov, steps, slices;
    float mu, keep, lr;
    char *x;           // [batch][slices][kSide][4 W]: the columns as they lie in LDS
    float *part;       // [2][batch][slices][kSide][kSide], by the step's parity
    int *exps;         // [batch][slices]
    int *lifts;        // [batch]
    int step;          // -1: the first launch; else a step (more than one slice)
};

// A matrix in LDS: rows of RS bytes, 8 hi, 8 lo, 8 hi, ...; a row's chunks change places by its last four bits, so that 16 rows' equal
// chunks are in different banks.
__device__ __forceinline__ uint32_t place(int row, int chunk, int rs) { return row * rs + ((chunk ^ (row & 15)) << 4); }

__device__ __forceinline__ void put(unsigned char *m, int rs, int row, int n, const float (&v)[4])
{
    union { _Float16 h[4]; u32x2 u; } hi, lo;
#pragma unroll
    for (int e = 0; e < 4; ++e) split_float(v[e], &hi.h[e], &lo.h[e]);
    const int c = (n >> 3) * 2, at = (n & 4) * 2;
    *(u32x2 *)(m + place(row, c, rs) + at) = hi.u;
    *(u32x2 *)(m + place(row, c + 1, rs) + at) = lo.u;
}
__device__ __forceinline__ void get(const unsigned char *m, int rs, int row, int n, float (&v)[4])
{
    union { _Float16 h[4]; u32x2 u; } hi, lo;
    const int c = (n >> 3) * 2, at = (n & 4) * 2;
    hi.u = *(const u32x2 *)(m + place(row, c, rs) + at);
    lo.u = *(const u32x2 *)(m + place(row, c + 1, rs) + at);
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = (float)hi.h[e] + (float)lo.h[e];
}
// fragments: 32 rows from row0 on, 16 terms along them from 16 s on ...
__device__ __forceinline__ s16x8 along(const unsigned char *m, int rs, int row0, int s, int part, int lane)
{
    return *(const s16x8 *)(m + place(row0 + (lane & 31), (s * 2 + (lane >> 5)) * 2 + part, rs));
}
// ... or 32 columns from col0 on, 16 terms down them
__device__ __forceinline__ s16x8 down(const unsigned char *m, int rs, int col0, int s, int part, int lane)
{
    typedef __attribute__((address_space(3))) s16x4 lds4;
    const int row = s * 16 + 8 * (lane >> 5) + ((lane & 15) >> 2);
    const int chunk = ((col0 + ((lane >> 4) & 1) * 16 + (lane & 3) * 4) >> 3) * 2 + part, at = (lane & 1) * 8;
    const uint32_t base = (uint32_t)(uintptr_t)(const __attribute__((address_space(3))) unsigned char *)m;
    union { s16x4 h[2]; s16x8 v; } r;
    r.h[0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4 *)(uintptr_t)(base + place(row, chunk, rs) + at));
    r.h[1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4 *)(uintptr_t)(base + place(row + 4, chunk, rs) + at));
    return r.v;
}
// A product is the sum of those with lo and then of the others: the first are 2^-11 of it and round by as much less (64 x 64: 1.4e-6 off, as
// float arithmetic is, and 1.7e-6 term by term).
__device__ __forceinline__ void two(s16x8 ah, s16x8 al, s16x8 bh, s16x8 bl, f32x16 *acc)
{
    *acc = product<Split>(bl, ah, *acc);
    *acc = product<Split>(bh, al, *acc);
}
__device__ __forceinline__ f32x16 zeros()
{
    f32x16 z;
#pragma unroll
    for (int r = 0; r < 16; ++r) z[r] = 0.f;
    return z;
}
// a value of every thread's, added up over the block in a fixed order, or the largest (red: a float a wave that nobody else uses)
template <bool LARGEST, int kWaves> __device__ __forceinline__ float over_block(float v, float *red)
{
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) v = LARGEST ? fmaxf(v, __shfl_xor(v, off, 64)) : v + __shfl_xor(v, off, 64);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
    __syncthreads();
    v = red[0];
#pragma unroll
    for (int w = 1; w < kWaves; ++w) v = LARGEST ? fmaxf(v, red[w]) : v + red[w];
    __syncthreads();
    return v;
}

// W columns to a workgroup of KG groups of 2 x 2 waves, which share the terms of X X^T
template <typename TG, typename TO, bool UPDATE, int W, int KG> __global__ void __launch_bounds__(256 * KG) narrow_kernel(const Args p)
{
    constexpr int kWaves = 4 * KG, kThreads = 64 * kWaves;
    extern __shared__ __align__(1024) unsigned char smem[];
    constexpr int RS = 4 * W, kCols = kSide * RS; // bytes
    constexpr int kOwn = W * 8 / kThreads;        // chunks of eight columns that a thread brings in
    constexpr int kApart = kWaves / 2, kJobs = W / 32 / kApart; // a wave multiplies every kApart-th block of 32 columns
    constexpr int kCopies = kCols / (16 * kThreads), kSums = 1024 / kThreads;
    unsigned char *X = smem, *A = smem + kCols, *B = A + kSquare;
    float *red = (float *)A;
    const int tid = threadIdx.x, wave = tid >> 6, group = wave >> 2, wm = (wave >> 1) & 1, wn = wave & 1;
    const int rb = (wave & 1) * 32, cb = wave >> 1; // the rows, and the first block of columns, of the polynomial's product
    const int slice = blockIdx.x, batch = blockIdx.y, j0 = slice * W;
    int lane = tid & 63;
    const long size = (long)p.r * p.n;
    char *x_mine = p.x + ((long)batch * p.slices + slice) * kCols;
    const bool single = p.slices == 1;

    int e_mine = 0, lift = 0;
    float ratio = 1.f; // what X has to be multiplied by to be X times kStore
    f32x16 s = zeros();

    auto gram = [&]() { // into the first group's s; A is free
        s = zeros();
        if (W > 64) asm volatile("" : "+v"(lane));
        constexpr int kSteps = W / 16 / KG;
#pragma unroll
        for (int kk = 0; kk < kSteps; ++kk) {
            const int k = kk * KG + group;
            two(along(X, RS, wm * 32, k, 0, lane), along(X, RS, wm * 32, k, 1, lane), along(X, RS, wn * 32, k, 0, lane), along(X, RS, wn * 32, k, 1, lane), &s);
        }
#pragma unroll
        for (int kk = 0; kk < kSteps; ++kk) {
            const int k = kk * KG + group;
            s = product<Split>(along(X, RS, wn * 32, k, 0, lane), along(X, RS, wm * 32, k, 0, lane), s);
        }
        if (KG == 1) return;
        f32x4 *sums = (f32x4 *)A + (wave & 3) * 256 + lane;
        if (group == 1)
#pragma unroll
            for (int q = 0; q < 4; ++q) sums[q * 64] = f32x4{s[q * 4], s[q * 4 + 1], s[q * 4 + 2], s[q * 4 + 3]};
        __syncthreads();
        if (group == 0)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const f32x4 v = sums[q * 64];
#pragma unroll
                for (int k = 0; k < 4; ++k) s[q * 4 + k] += v[k];
            }
        __syncthreads();
    };
    auto leave = [&](int parity) { // this workgroup's part of X X^T, and its columns
        float *o = p.part + ((((long)parity * gridDim.y + batch) * p.slices) + slice) * (kSide * kSide);
        if (group == 0)
#pragma unroll
            for (int q = 0; q < 4; ++q)
                *(f32x4 *)(o + (wm * 32 + (lane & 31)) * kSide + wn * 32 + q * 8 + (lane >> 5) * 4) = f32x4{s[q * 4], s[q * 4 + 1], s[q * 4 + 2], s[q * 4 + 3]};
#pragma unroll
        for (int c = 0; c < kCopies; ++c) *(u32x4 *)(x_mine + (c * kThreads + tid) * 16) = *(const u32x4 *)(X + (c * kThreads + tid) * 16);
    };

    if (p.step < 0) {
        // U, eight neighbouring columns of a row to a thread and turn; neighbouring threads take neighbours in memory.  A few turns' numbers
        // are asked for before any is stored, so that they are on their way together.  Until the largest number is known they wait as
        // floats where their halves will be.
        float top = 0.f;
        const TG *g = (const TG *)p.G + batch * size;
        float *m = p.M ? p.M + batch * size : nullptr;
        // (rows of whole groups of four, and a first column that is one of 64: four neighbours in one access)
        const bool wide = !p.tall && (p.n & 3) == 0;
        struct alignas(4 * sizeof(TG)) Four { TG v[4]; };
        constexpr int kTogether = kOwn <= 4 ? kOwn : 4;
        auto row_of = [&](int c) { return p.tall ? (c * kThreads + tid) & 63 : (c * kThreads + tid) / (W / 8); };
        auto col_of = [&](int c) { return (p.tall ? (c * kThreads + tid) >> 6 : (c * kThreads + tid) % (W / 8)) * 8; };
#pragma unroll 1
        for (int c0 = 0; c0 < kOwn; c0 += kTogether) {
            float u[kTogether][8], mm[kTogether][8];
#pragma unroll
            for (int t = 0; t < kTogether; ++t) {
                const int i = row_of(c0 + t), j = j0 + col_of(c0 + t);
                const long at = p.tall ? (long)j * p.r + i : (long)i * p.n + j, step = p.tall ? p.r : 1;
                const int left = i < p.r ? p.n - j : 0; // elements from the first on
#pragma unroll
                for (int h = 0; h < 8; h += 4) {
                    if (wide) {
                        Four f;
                        f32x4 o = {0.f, 0.f, 0.f, 0.f};
                        if (h < left) f = *(const Four *)(g + at + h);
                        if (h < left && m) o = *(const f32x4 *)(m + at + h);
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            u[t][h + e] = h < left ? Elem<TG>::load(&f.v[e]) : 0.f;
                            mm[t][h + e] = o[e];
                        }
                    } else {
#pragma unroll
                        for (int e = h; e < h + 4; ++e) {
                            u[t][e] = e < left ? Elem<TG>::load(g + at + e * step) : 0.f;
                            mm[t][e] = e < left && m ? m[at + e * step] : 0.f;
                        }
                    }
                }
            }
#pragma unroll
            for (int t = 0; t < kTogether; ++t) {
                const int i = row_of(c0 + t), jc = col_of(c0 + t), j = j0 + jc;
                const long at = p.tall ? (long)j * p.r + i : (long)i * p.n + j, step = p.tall ? p.r : 1;
                const int left = i < p.r ? p.n - j : 0;
                if (m) {
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        mm[t][e] = p.mu * mm[t][e] + u[t][e];
                        u[t][e] = p.nesterov ? u[t][e] + p.mu * mm[t][e] : mm[t][e];
                    }
#pragma unroll
                    for (int h = 0; h < 8; h += 4) {
                        if (wide) {
                            if (h < left) *(f32x4 *)(m + at + h) = f32x4{mm[t][h], mm[t][h + 1], mm[t][h + 2], mm[t][h + 3]};
                        } else {
#pragma unroll
                            for (int e = h; e < h + 4; ++e)
                                if (e < left) m[at + e * step] = mm[t][e];
                        }
                    }
                }
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const float a = fabsf(u[t][e]);
                    top = a <= 3.4028235e38f ? fmaxf(top, a) : top;
                }
#pragma unroll
                for (int h = 0; h < 2; ++h)
                    *(f32x4 *)(X + place(i, (jc >> 3) * 2 + h, RS)) = f32x4{u[t][h * 4], u[t][h * 4 + 1], u[t][h * 4 + 2], u[t][h * 4 + 3]};
            }
        }
        top = over_block<true, kWaves>(top, red);
        if (top > 0.f) {
            frexpf(top, &e_mine);
            e_mine = 12 - e_mine; // the largest is stored as one below 2^12
        } else {
            e_mine = kNone;
        }
#pragma unroll 1
        for (int c = 0; c < kOwn; ++c) {
            const int i = row_of(c), jc = col_of(c);
            const f32x4 a = *(const f32x4 *)(X + place(i, (jc >> 3) * 2, RS)), b = *(const f32x4 *)(X + place(i, (jc >> 3) * 2 + 1, RS));
            const float v[4] = {ldexpf(a[0], e_mine), ldexpf(a[1], e_mine), ldexpf(a[2], e_mine), ldexpf(a[3], e_mine)};
            const float w[4] = {ldexpf(b[0], e_mine), ldexpf(b[1], e_mine), ldexpf(b[2], e_mine), ldexpf(b[3], e_mine)};
            put(X, RS, i, jc, v);
            put(X, RS, i, jc + 4, w);
        }
        __syncthreads();
        gram();
        if (!single) {
            leave(0);
            if (tid == 0) p.exps[batch * p.slices + slice] = e_mine;
            return;
        }
    }

    const int first = single ? 0 : p.step, last = single ? p.steps : p.step + 1;
    for (int step = first; step < last; ++step) {
        if (W > 64) asm volatile("" : "+v"(lane)); // (places in LDS are worked out where they are used: kept from step to step they take all registers)
        // A times kStore, as two halves
        if (single) {
            float take = ldexpf(kTake, -2 * lift);
            if (step == 0) {
                float d = 0.f;
                if (group == 0 && wm == wn)
#pragma unroll
                    for (int q = 0; q < 4; ++q)
#pragma unroll
                        for (int k = 0; k < 4; ++k)
                            if (q * 8 + (lane >> 5) * 4 + k == (lane & 31)) d += s[q * 4 + k];
                const double size = sqrt((double)over_block<false, kWaves>(d, red)), norm = size + ldexp((double)kNsEps, e_mine); // times 2^e_mine
                lift = ns_lift(ldexp(size, -e_mine), p.steps);
                ratio = (float)(ldexp((double)kStore, lift) / norm);
                take = (float)((double)kStore / (norm * norm));
            }
            if (group == 0)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const float v[4] = {s[q * 4] * take, s[q * 4 + 1] * take, s[q * 4 + 2] * take, s[q * 4 + 3] * take};
                put(A, 256, wm * 32 + (lane & 31), wn * 32 + q * 8 + (lane >> 5) * 4, v);
            }
        } else {
            const float *part = p.part + ((long)(step & 1) * gridDim.y + batch) * p.slices * (kSide * kSide);
            const int *exps = p.exps + batch * p.slices;
            // the slices' powers of two are brought to that of the largest numbers (a lane knows one slice's: there are at most 64)
            int e_ref = step == 0 ? exps[min(lane, p.slices - 1)] : 0;
            const int e_lane = e_ref;
#pragma unroll
            for (int off = 32; off > 0; off >>= 1) e_ref = min(e_ref, __shfl_xor(e_ref, off, 64));
            u32x4 mine[kCopies]; // (the columns are on their way while the parts are added up)
#pragma unroll
            for (int c = 0; c < kCopies; ++c) mine[c] = *(const u32x4 *)(x_mine + (c * kThreads + tid) * 16);
            float v[kSums][4] = {};
            for (int k0 = 0; k0 < p.slices; k0 += 16 / kSums) { // sixteen accesses on their way at a time
                f32x4 x[16 / kSums][kSums];
#pragma unroll
                for (int k = 0; k < 16 / kSums; ++k)
#pragma unroll
                    for (int c = 0; c < kSums; ++c)
                        x[k][c] = k0 + k < p.slices && c * (kThreads / 16) + (tid >> 4) < p.r ? *(const f32x4 *)(part + (long)(k0 + k) * (kSide * kSide) + (c * kThreads + tid) * 4) : f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int k = 0; k < 16 / kSums; ++k) {
                    const float w = ldexpf(1.f, 2 * (e_ref - __shfl(e_lane, min(k0 + k, p.slices - 1), 64)));
#pragma unroll
                    for (int c = 0; c < kSums; ++c)
#pragma unroll
                        for (int e = 0; e < 4; ++e) v[c][e] += w * x[k][c][e];
                }
            }
#pragma unroll
            for (int c = 0; c < kCopies; ++c) *(u32x4 *)(X + (c * kThreads + tid) * 16) = mine[c];
            if (step > 0) lift = p.lifts[batch];
            float take = ldexpf(kTake, -2 * lift);
            if (step == 0) {
                float d = 0.f;
#pragma unroll
                for (int c = 0; c < kSums; ++c)
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        if ((tid & 15) * 4 + e == c * (kThreads / 16) + (tid >> 4)) d += v[c][e];
                const double size = sqrt((double)over_block<false, kWaves>(d, red)), norm = size + ldexp((double)kNsEps, e_ref); // times 2^e_ref
                lift = ns_lift(ldexp(size, -e_ref), p.steps);
                if (slice == 0 && tid == 0) p.lifts[batch] = lift;
                ratio = (float)(ldexp((double)kStore, e_ref - exps[slice] + lift) / norm);
                take = (float)((double)kStore / (norm * norm));
            }
#pragma unroll
            for (int c = 0; c < kSums; ++c) {
#pragma unroll
                for (int e = 0; e < 4; ++e) v[c][e] *= take;
                put(A, 256, c * (kThreads / 16) + (tid >> 4), (tid & 15) * 4, v[c]);
            }
        }
        __syncthreads();
        // a I + b A + c A A, by the first group
        if (group == 0) {
            f32x16 acc = zeros();
#pragma unroll
            for (int k = 0; k < kSide / 16; ++k)
                two(along(A, 256, wm * 32, k, 0, lane), along(A, 256, wm * 32, k, 1, lane), along(A, 256, wn * 32, k, 0, lane), along(A, 256, wn * 32, k, 1, lane), &acc);
#pragma unroll
            for (int k = 0; k < kSide / 16; ++k) acc = product<Split>(along(A, 256, wn * 32, k, 0, lane), along(A, 256, wm * 32, k, 0, lane), acc);
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const int i = wm * 32 + (lane & 31), j = wn * 32 + q * 8 + (lane >> 5) * 4;
                float v[4];
                get(A, 256, i, j, v);
#pragma unroll
                for (int k = 0; k < 4; ++k) v[k] = kB * v[k] + (kC * kTake) * acc[q * 4 + k] + (i == j + k ? kA * kStore : 0.f);
                put(B, 256, i, j, v);
            }
        }
        __syncthreads();
        // ... times X: 32 rows, every kApart-th block of columns
        if (W > 64) asm volatile("" : "+v"(lane));
        f32x16 y[kJobs];
#pragma unroll
        for (int b = 0; b < kJobs; ++b) y[b] = zeros();
#pragma unroll
        for (int k = 0; k < kSide / 16; ++k) {
            const s16x8 ph = along(B, 256, rb, k, 0, lane), pl = along(B, 256, rb, k, 1, lane);
#pragma unroll
            for (int b = 0; b < kJobs; ++b)
                two(ph, pl, down(X, RS, (cb + b * kApart) * 32, k, 0, lane), down(X, RS, (cb + b * kApart) * 32, k, 1, lane), &y[b]);
        }
#pragma unroll
        for (int k = 0; k < kSide / 16; ++k) {
            const s16x8 ph = along(B, 256, rb, k, 0, lane);
#pragma unroll
            for (int b = 0; b < kJobs; ++b) y[b] = product<Split>(down(X, RS, (cb + b * kApart) * 32, k, 0, lane), ph, y[b]);
        }
        if (step + 1 == p.steps) {
            const float scale = ldexpf((UPDATE ? -p.lr : 1.f) * kTake * kTake * ratio, -lift);
            TO *out = (TO *)p.out + batch * size;
            const int i = rb + (lane & 31);
            auto where = [&](int b, int q, int k) -> long {
                const int j = j0 + (cb + b * kApart) * 32 + q * 8 + (lane >> 5) * 4 + k;
                if (i >= p.r || j >= p.n) return -1;
                return p.tall ? (long)j * p.r + i : (long)i * p.n + j;
            };
            const bool wide = !p.tall && (p.n & 3) == 0;
            struct alignas(4 * sizeof(TO)) Four { TO v[4]; };
#pragma unroll
            for (int b = 0; b < kJobs; ++b) {
                float old[16] = {};
                if (UPDATE) { // (asked for together, before the first store)
#pragma unroll
                    for (int q = 0; q < 4; ++q)
                        if (wide) {
                            const long at = where(b, q, 0);
                            Four f;
                            if (at >= 0) f = *(const Four *)(out + at);
#pragma unroll
                            for (int k = 0; k < 4; ++k) old[q * 4 + k] = at >= 0 ? Elem<TO>::load(&f.v[k]) : 0.f;
                        } else {
#pragma unroll
                            for (int k = 0; k < 4; ++k) {
                                const long at = where(b, q, k);
                                old[q * 4 + k] = at >= 0 ? Elem<TO>::load(out + at) : 0.f;
                            }
                        }
                }
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    float v[4];
#pragma unroll
                    for (int k = 0; k < 4; ++k) v[k] = UPDATE ? p.keep * old[q * 4 + k] + scale * y[b][q * 4 + k] : scale * y[b][q * 4 + k];
                    if (wide) {
                        const long at = where(b, q, 0);
                        Four f;
#pragma unroll
                        for (int k = 0; k < 4; ++k) Elem<TO>::store(&f.v[k], v[k]);
                        if (at >= 0) *(Four *)(out + at) = f;
                    } else {
#pragma unroll
                        for (int k = 0; k < 4; ++k) {
                            const long at = where(b, q, k);
                            if (at >= 0) Elem<TO>::store(out + at, v[k]);
                        }
                    }
                }
            }
            return;
        }
        __syncthreads(); // (every wave has read the columns that it multiplied)
        if (W > 64) asm volatile("" : "+v"(lane));
#pragma unroll
        for (int b = 0; b < kJobs; ++b)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                float v[4];
#pragma unroll
                for (int k = 0; k < 4; ++k) v[k] = y[b][q * 4 + k] * (kTake * ratio);
                put(X, RS, rb + (lane & 31), (cb + b * kApart) * 32 + q * 8 + (lane >> 5) * 4, v);
            }
        ratio = 1.f;
        __syncthreads();
        gram();
        if (!single) leave((step + 1) & 1);
    }
}

size_t up(size_t n) { return (n + 255) & ~(size_t)255; }

template <typename TG, typename TO, bool UPDATE, int W, int KG> hipError_t launch(Args a, int batch, hipStream_t st)
{
    constexpr int lds = kSide * 4 * W + 2 * kSquare;
    static const hipError_t attr = hipFuncSetAttribute(reinterpret_cast<const void *>(narrow_kernel<TG, TO, UPDATE, W, KG>),
                                                       hipFuncAttributeMaxDynamicSharedMemorySize, lds);
    if (attr != hipSuccess) return attr;
    for (int step = -1; step < (a.slices == 1 ? 0 : a.steps); ++step) {
        a.step = step;
        hipLaunchKernelGGL((narrow_kernel<TG, TO, UPDATE, W, KG>), dim3(a.slices, batch), dim3(256 * KG), lds, st, a);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}
template <typename TG, typename TO, bool UPDATE> hipError_t launch(const Args &a, int width, int batch, hipStream_t st)
{
    if (width == 64) return launch<TG, TO, UPDATE, 64, 1>(a, batch, st);
    if (width == 128) return launch<TG, TO, UPDATE, 128, 1>(a, batch, st);
    return launch<TG, TO, UPDATE, 256, 2>(a, batch, st);
}
template <typename TG> hipError_t launch(const Args &a, int width, int batch, int dtype, bool update, hipStream_t st)
{
    if (dtype == CAC_F32) return update ? launch<TG, float, true>(a, width, batch, st) : launch<TG, float, false>(a, width, batch, st);
    return update ? launch<TG, bf16_t, true>(a, width, batch, st) : launch<TG, bf16_t, false>(a, width, batch, st);
}

} // namespace

bool plan_muon_narrow(const MuonGeom &g, MuonNarrowPlan *p)
{
    const long r = g.rows < g.cols ? g.rows : g.cols, n = g.rows < g.cols ? g.cols : g.rows;
    // Every workgroup reads all of its matrix' parts, and a lane knows one part's power of two: not more than 64 of them (64 x 16384: 108 us
    // here, 148 with muon.hip's launches; 64 x 2048 60 and 93).
    if (r > kSide || n > 16384) return false;
    // The narrowest that holds a matrix in one launch; else more workgroups while their parts are few (a step of 64 x 576 in columns of 64,
    // 128 and 256: 55, 52 and 57 us, of 64 x 2048 81, 64 and 60, of 64 x 8192 -, 128 and 80).
    p->width = n <= 64 ? 64 : n <= 128 ? 128 : n <= 256 ? 256 : n <= 1024 ? 128 : 256;
    p->slices = (int)((n + p->width - 1) / p->width);
    size_t o = 0;
    p->o_x = o;
    if (p->slices > 1) o += up((size_t)g.batch * p->slices * kSide * 4 * p->width);
    p->o_part = o;
    if (p->slices > 1) o += up((size_t)2 * g.batch * p->slices * kSide * kSide * 4);
    p->o_exps = o;
    if (p->slices > 1) o += up((size_t)g.batch * (p->slices + 1) * 4);
    p->bytes = o;
    return true;
}

hipError_t launch_muon_narrow(const MuonGeom &g, const MuonNarrowPlan &p, const void *G, float *M, void *W, void *O, float momentum, float keep,
                              float lr, void *ws_, hipStream_t st)
{
    char *ws = (char *)ws_;
    Args a{};
    a.G = G;
    a.M = M;
    a.out = W ? W : O;
    a.tall = g.rows > g.cols;
    a.r = (int)(a.tall ? g.cols : g.rows);
    a.n = (int)(a.tall ? g.rows : g.cols);
    a.nesterov = g.nesterov;
    a.steps = g.steps;
    a.slices = p.slices;
    a.mu = momentum;
    a.keep = keep;
    a.lr = lr;
    a.x = ws + p.o_x;
    a.part = (float *)(ws + p.o_part);
    a.exps = (int *)(ws + p.o_exps);
    a.lifts = a.exps + (size_t)g.batch * p.slices;
    if (g.grad_dtype == CAC_F32) return launch<float>(a, p.width, g.batch, g.dtype, W != nullptr, st);
    return launch<bf16_t>(a, p.width, g.batch, g.dtype, W != nullptr, st);
}

} // namespace cac
