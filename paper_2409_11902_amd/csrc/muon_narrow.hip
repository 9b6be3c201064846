// The orthogonalised update (muon.hip) of matrices whose shorter side is at most 64: what takes time there is launches, not products.
//
// A workgroup owns 64, 128 or 256 columns of its matrix (rows and columns are the shorter and the longer side here) as two halves in
// LDS, and the square products of 64 x 64 are cheap enough for every workgroup to form the polynomial by itself.  A matrix that one
// workgroup holds is done in one launch; a longer one takes a launch a step, which adds up the workgroups' parts of X X^T, forms the
// polynomial, multiplies its columns by it and leaves its part of the next X X^T.  No launch is spent on the norm: it is the
// trace of U U^T, and a workgroup's columns of U are stored times a power of two of their own until it is known.
#include "mm_core.h"

namespace cac {

namespace {

using namespace mm;

constexpr float kA = 3.4445f, kB = -4.7750f, kC = 2.0315f, kEps = 1e-7f;
constexpr float kStore = 4096.f, kTake = 1.f / 4096.f; // what X, A and the polynomial are stored times
constexpr int kSide = 64, kSquare = kSide * 256;       // bytes of a square matrix in LDS

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
__device__ __forceinline__ void three(s16x8 ah, s16x8 al, s16x8 bh, s16x8 bl, f32x16 *acc)
{
    *acc = product<Split>(bh, ah, *acc);
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
// a value of every thread's, added up over the block in a fixed order (red: 4 floats)
__device__ __forceinline__ float block_sum(float v, float *red)
{
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) v += __shfl_xor(v, off, 64);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
    __syncthreads();
    return ((red[0] + red[1]) + red[2]) + red[3];
}

// W columns to a workgroup of four waves
template <typename TG, typename TO, bool UPDATE, int W> __global__ void __launch_bounds__(256) narrow_kernel(const Args p)
{
    extern __shared__ __align__(1024) unsigned char smem[];
    constexpr int RS = 4 * W, kCols = kSide * RS; // bytes
    constexpr int kOwn = W / 32;                  // chunks of eight columns that a thread brings in
    constexpr int kJobs = W / 64;                 // blocks of 32 x 32 that a wave multiplies
    unsigned char *X = smem, *A = smem + kCols, *B = A + kSquare;
    float *red = (float *)(B + kSquare);
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, wm = wave >> 1, wn = wave & 1;
    const int slice = blockIdx.x, batch = blockIdx.y, j0 = slice * W;
    const long size = (long)p.r * p.n;
    char *x_mine = p.x + ((long)batch * p.slices + slice) * kCols;
    const bool single = p.slices == 1;

    int e_mine = 0;
    float ratio = 1.f; // what X has to be multiplied by to be X times kStore
    f32x16 s = zeros();

    auto gram = [&]() {
        s = zeros();
#pragma unroll 4
        for (int k = 0; k < W / 16; ++k)
            three(along(X, RS, wm * 32, k, 0, lane), along(X, RS, wm * 32, k, 1, lane), along(X, RS, wn * 32, k, 0, lane), along(X, RS, wn * 32, k, 1, lane), &s);
    };
    auto leave = [&](int parity) { // this workgroup's part of X X^T, and its columns
        float *o = p.part + ((((long)parity * gridDim.y + batch) * p.slices) + slice) * (kSide * kSide);
#pragma unroll
        for (int q = 0; q < 4; ++q)
            *(f32x4 *)(o + (wm * 32 + (lane & 31)) * kSide + wn * 32 + q * 8 + (lane >> 5) * 4) = f32x4{s[q * 4], s[q * 4 + 1], s[q * 4 + 2], s[q * 4 + 3]};
        for (int c = tid * 16; c < kCols; c += 4096) *(u32x4 *)(x_mine + c) = *(const u32x4 *)(X + c);
    };

    if (p.step < 0) {
        // U, eight neighbouring columns of a row to a thread and turn; neighbouring threads take neighbours in memory.  Everything is
        // asked for before anything is stored, so that it is on its way together.
        float u[kOwn][8], top = 0.f;
        const TG *g = (const TG *)p.G + batch * size;
        float *m = p.M ? p.M + batch * size : nullptr;
        auto where = [&](int c, int e) -> long { // of element e of turn c; -1 past the edge
            const int at = c * 256 + tid, i = p.tall ? at & 63 : at / (W / 8), j = j0 + (p.tall ? at >> 6 : at % (W / 8)) * 8 + e;
            if (i >= p.r || j >= p.n) return -1;
            return p.tall ? (long)j * p.r + i : (long)i * p.n + j;
        };
        // (rows of whole groups of four, and a first column that is one of 64: four neighbours in one access)
        const bool wide = !p.tall && (p.n & 3) == 0;
        struct alignas(4 * sizeof(TG)) Four { TG v[4]; };
#pragma unroll
        for (int c = 0; c < kOwn; ++c) {
            if (wide) {
#pragma unroll
                for (int h = 0; h < 8; h += 4) {
                    const long k = where(c, h);
                    Four f;
                    if (k >= 0) f = *(const Four *)(g + k);
#pragma unroll
                    for (int e = 0; e < 4; ++e) u[c][h + e] = k >= 0 ? Elem<TG>::load(&f.v[e]) : 0.f;
                }
            } else {
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const long k = where(c, e);
                    u[c][e] = k >= 0 ? Elem<TG>::load(g + k) : 0.f;
                }
            }
        }
        if (m) {
            float mm[kOwn][8];
#pragma unroll
            for (int c = 0; c < kOwn; ++c)
                if (wide) {
#pragma unroll
                    for (int h = 0; h < 8; h += 4) {
                        const long k = where(c, h);
                        const f32x4 f = k >= 0 ? *(const f32x4 *)(m + k) : f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                        for (int e = 0; e < 4; ++e) mm[c][h + e] = f[e];
                    }
                } else {
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        const long k = where(c, e);
                        mm[c][e] = k >= 0 ? m[k] : 0.f;
                    }
                }
#pragma unroll
            for (int c = 0; c < kOwn; ++c) {
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    mm[c][e] = p.mu * mm[c][e] + u[c][e];
                    u[c][e] = p.nesterov ? u[c][e] + p.mu * mm[c][e] : mm[c][e];
                }
                if (wide) {
#pragma unroll
                    for (int h = 0; h < 8; h += 4) {
                        const long k = where(c, h);
                        if (k >= 0) *(f32x4 *)(m + k) = f32x4{mm[c][h], mm[c][h + 1], mm[c][h + 2], mm[c][h + 3]};
                    }
                } else {
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        const long k = where(c, e);
                        if (k >= 0) m[k] = mm[c][e];
                    }
                }
            }
        }
#pragma unroll
        for (int c = 0; c < kOwn; ++c)
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float a = fabsf(u[c][e]);
                top = a <= 3.4028235e38f ? fmaxf(top, a) : top;
            }
#pragma unroll
        for (int off = 32; off > 0; off >>= 1) top = fmaxf(top, __shfl_xor(top, off, 64));
        if (lane == 0) red[wave] = top;
        __syncthreads();
        top = fmaxf(fmaxf(red[0], red[1]), fmaxf(red[2], red[3]));
        if (top > 0.f) {
            frexpf(top, &e_mine);
            e_mine = 12 - e_mine; // the largest is stored as one below 2^12
        }
#pragma unroll
        for (int c = 0; c < kOwn; ++c) {
            const int at = c * 256 + tid, i = p.tall ? at & 63 : at / (W / 8), j = (p.tall ? at >> 6 : at % (W / 8)) * 8;
#pragma unroll
            for (int h = 0; h < 8; h += 4) {
                const float v[4] = {ldexpf(u[c][h], e_mine), ldexpf(u[c][h + 1], e_mine), ldexpf(u[c][h + 2], e_mine), ldexpf(u[c][h + 3], e_mine)};
                put(X, RS, i, j + h, v);
            }
        }
        __syncthreads();
        gram();
        if (!single) {
            leave(0);
            if (tid == 0) p.exps[batch * p.slices + slice] = e_mine;
            return;
        }
    } else {
        u32x4 x[kCols / 4096];
#pragma unroll
        for (int c = 0; c < kCols / 4096; ++c) x[c] = *(const u32x4 *)(x_mine + c * 4096 + tid * 16);
#pragma unroll
        for (int c = 0; c < kCols / 4096; ++c) *(u32x4 *)(X + c * 4096 + tid * 16) = x[c];
    }

    const int first = single ? 0 : p.step, last = single ? p.steps : p.step + 1;
    for (int step = first; step < last; ++step) {
        // A times kStore, as two halves
        if (single) {
            float take = kTake;
            if (step == 0) {
                float d = 0.f;
                if (wm == wn)
#pragma unroll
                    for (int q = 0; q < 4; ++q)
#pragma unroll
                        for (int k = 0; k < 4; ++k)
                            if (q * 8 + (lane >> 5) * 4 + k == (lane & 31)) d += s[q * 4 + k];
                const double norm = sqrt((double)block_sum(d, red)) + ldexp((double)kEps, e_mine); // in U's units times 2^e_mine
                ratio = (float)((double)kStore / norm);
                take = (float)((double)kStore / (norm * norm));
            }
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const float v[4] = {s[q * 4] * take, s[q * 4 + 1] * take, s[q * 4 + 2] * take, s[q * 4 + 3] * take};
                put(A, 256, wm * 32 + (lane & 31), wn * 32 + q * 8 + (lane >> 5) * 4, v);
            }
        } else {
            const float *part = p.part + ((long)(step & 1) * gridDim.y + batch) * p.slices * (kSide * kSide);
            const int *exps = p.exps + batch * p.slices;
            // the slices' powers of two are brought to that of the largest numbers (a lane knows one slice's: there are at most 32)
            int e_ref = step == 0 ? exps[min(lane, p.slices - 1)] : 0;
            const int e_lane = e_ref;
#pragma unroll
            for (int off = 32; off > 0; off >>= 1) e_ref = min(e_ref, __shfl_xor(e_ref, off, 64));
            float v[4][4] = {};
            for (int k0 = 0; k0 < p.slices; k0 += 4) { // sixteen accesses on their way at a time
                f32x4 x[4][4];
#pragma unroll
                for (int k = 0; k < 4; ++k)
#pragma unroll
                    for (int c = 0; c < 4; ++c)
                        x[k][c] = k0 + k < p.slices ? *(const f32x4 *)(part + (long)(k0 + k) * (kSide * kSide) + c * 1024 + tid * 4) : f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    const float w = ldexpf(1.f, 2 * (e_ref - __shfl(e_lane, min(k0 + k, p.slices - 1), 64)));
#pragma unroll
                    for (int c = 0; c < 4; ++c)
#pragma unroll
                        for (int e = 0; e < 4; ++e) v[c][e] += w * x[k][c][e];
                }
            }
            float take = kTake;
            if (step == 0) {
                float d = 0.f;
#pragma unroll
                for (int c = 0; c < 4; ++c)
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        if ((tid & 15) * 4 + e == c * 16 + (tid >> 4)) d += v[c][e];
                const double norm = sqrt((double)block_sum(d, red)) + ldexp((double)kEps, e_ref);
                ratio = (float)(ldexp((double)kStore, e_ref - exps[slice]) / norm);
                take = (float)((double)kStore / (norm * norm));
            }
#pragma unroll
            for (int c = 0; c < 4; ++c) {
#pragma unroll
                for (int e = 0; e < 4; ++e) v[c][e] *= take;
                put(A, 256, c * 16 + (tid >> 4), (tid & 15) * 4, v[c]);
            }
        }
        __syncthreads();
        // a I + b A + c A A
        f32x16 acc = zeros();
#pragma unroll
        for (int k = 0; k < kSide / 16; ++k)
            three(along(A, 256, wm * 32, k, 0, lane), along(A, 256, wm * 32, k, 1, lane), along(A, 256, wn * 32, k, 0, lane), along(A, 256, wn * 32, k, 1, lane), &acc);
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const int i = wm * 32 + (lane & 31), j = wn * 32 + q * 8 + (lane >> 5) * 4;
            float v[4];
            get(A, 256, i, j, v);
#pragma unroll
            for (int k = 0; k < 4; ++k) v[k] = kB * v[k] + (kC * kTake) * acc[q * 4 + k] + (i == j + k ? kA * kStore : 0.f);
            put(B, 256, i, j, v);
        }
        __syncthreads();
        // ... times X: rows wm * 32 on, every other block of columns
        f32x16 y[kJobs];
#pragma unroll
        for (int b = 0; b < kJobs; ++b) y[b] = zeros();
#pragma unroll
        for (int k = 0; k < kSide / 16; ++k) {
            const s16x8 bh = along(B, 256, wm * 32, k, 0, lane), bl = along(B, 256, wm * 32, k, 1, lane);
#pragma unroll
            for (int b = 0; b < kJobs; ++b)
                three(bh, bl, down(X, RS, (b * 2 + wn) * 32, k, 0, lane), down(X, RS, (b * 2 + wn) * 32, k, 1, lane), &y[b]);
        }
        if (step + 1 == p.steps) {
            const float scale = (UPDATE ? -p.lr : 1.f) * kTake * kTake * ratio;
            TO *out = (TO *)p.out + batch * size;
            const int i = wm * 32 + (lane & 31);
            auto where = [&](int b, int q, int k) -> long {
                const int j = j0 + (b * 2 + wn) * 32 + q * 8 + (lane >> 5) * 4 + k;
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
#pragma unroll
        for (int b = 0; b < kJobs; ++b)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                float v[4];
#pragma unroll
                for (int k = 0; k < 4; ++k) v[k] = y[b][q * 4 + k] * (kTake * ratio);
                put(X, RS, wm * 32 + (lane & 31), (b * 2 + wn) * 32 + q * 8 + (lane >> 5) * 4, v);
            }
        ratio = 1.f;
        __syncthreads();
        gram();
        if (!single) leave((step + 1) & 1);
    }
}

size_t up(size_t n) { return (n + 255) & ~(size_t)255; }

template <typename TG, typename TO, bool UPDATE, int W> hipError_t launch(Args a, int batch, hipStream_t st)
{
    constexpr int lds = kSide * 4 * W + 2 * kSquare + 64;
    static const hipError_t attr = hipFuncSetAttribute(reinterpret_cast<const void *>(narrow_kernel<TG, TO, UPDATE, W>),
                                                       hipFuncAttributeMaxDynamicSharedMemorySize, lds);
    if (attr != hipSuccess) return attr;
    for (int step = -1; step < (a.slices == 1 ? 0 : a.steps); ++step) {
        a.step = step;
        hipLaunchKernelGGL((narrow_kernel<TG, TO, UPDATE, W>), dim3(a.slices, batch), dim3(256), lds, st, a);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}
template <typename TG, typename TO, bool UPDATE> hipError_t launch(const Args &a, int width, int batch, hipStream_t st)
{
    if (width == 64) return launch<TG, TO, UPDATE, 64>(a, batch, st);
    if (width == 128) return launch<TG, TO, UPDATE, 128>(a, batch, st);
    return launch<TG, TO, UPDATE, 256>(a, batch, st);
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
    // every workgroup reads all of its matrix' parts: not more than 32 of them
    if (r > kSide || n > 8192) return false;
    p->width = n <= 64 ? 64 : n <= 128 || (n > 256 && n <= 2048) ? 128 : 256;
    p->slices = (int)((n + p->width - 1) / p->width);
    size_t o = 0;
    p->o_x = o;
    if (p->slices > 1) o += up((size_t)g.batch * p->slices * kSide * 4 * p->width);
    p->o_part = o;
    if (p->slices > 1) o += up((size_t)2 * g.batch * p->slices * kSide * kSide * 4);
    p->o_exps = o;
    if (p->slices > 1) o += up((size_t)g.batch * p->slices * 4);
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
    if (g.grad_dtype == CAC_F32) return launch<float>(a, p.width, g.batch, g.dtype, W != nullptr, st);
    return launch<bf16_t>(a, p.width, g.batch, g.dtype, W != nullptr, st);
}

} // namespace cac
