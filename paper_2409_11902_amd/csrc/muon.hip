// The orthogonalised form of a gradient, and the optimiser's step made of it.
//
//   X_0 = U / (|U|_F + 1e-7);  A = X X^T,  X <- (a I + b A + c A A) X, `steps` times
//
// with (a, b, c) = (3.4445, -4.7750, 2.0315), which drives every singular value towards 1 (within about 0.7 to 1.2) and keeps the
// singular vectors.  U is the gradient, or with momentum M <- mu M + G, U = G + mu M (U = M without nesterov) and afterwards
// W <- keep W - lr X.  A matrix of more rows than columns takes A = X^T X and X <- X (a I + b A + c A A): the square products are of
// the shorter side.
//
// Everything between U and the result is held as two halves (mm_core.h), times 2^12: the first products' errors are multiplied by up
// to a^steps (485 for five) in the directions that a gradient has least of, so 8 or 11 bits there end as 1e-2 of the result.
#include "mm_core.h"
#include "train_ends.h"

namespace cac {

namespace {

using namespace mm;

constexpr float kA = kNsA, kB = kNsB, kC = kNsC, kTake = kNsTake, kStore = kNsStore;
constexpr int kMaxSumBlocks = 256;

// ---- endings of the products
// S = acc / 4096, symmetric: the tiles above the diagonal are computed and written twice
struct Gram : Ending {
    static constexpr bool kSymmetric = true;
    struct Params { char *out; long ld, stride; const int *lift; };
    template <int MI, int NI> static __device__ __forceinline__ void run(const Params &e, const f32x16 (&acc)[MI][NI], const Place &p);
};
// a I + b A + c A A
struct Poly : Ending {
    static constexpr bool kSymmetric = true;
    struct Params { char *out; long ld, stride; const char *a; };
    template <int MI, int NI> static __device__ __forceinline__ void run(const Params &e, const f32x16 (&acc)[MI][NI], const Place &p);
};

// v of row m, columns n..n+3 of a symmetric matrix, to its place and, off the diagonal tiles, to the mirrored one
__device__ __forceinline__ void store_symmetric(char *out, long ld, int m, int n, int M, int Np, bool mirror, const float (&v)[4])
{
    if (m < M && n < Np) store_split(out + m * ld, n, v);
    if (!mirror) return;
    if (m >= Np) return;
#pragma unroll
    for (int e = 0; e < 4; ++e)
        if (n + e < M) {
            _Float16 hi, lo;
            split_float(v[e], &hi, &lo);
            char *c = out + (n + e) * ld + (m >> 3) * 32 + (m & 7) * 2;
            *(_Float16 *)c = hi;
            *(_Float16 *)(c + 16) = lo;
        }
}
// a wave's part of a symmetric matrix, value(i, j, q, m, n, v) giving four of it
template <int MI, int NI, class Fn> __device__ __forceinline__ void store_symmetric_part(char *out, long ld, const Place &p, Fn value)
{
    const int Np = (p.N + 7) & ~7;
    typedef RowBlock<Fmt::kSplit, 1> Block;
#pragma unroll
    for (int i = 0; i < MI; ++i)
#pragma unroll
        for (int j = 0; j < NI; ++j) {
            const int m0 = p.m0 + i * 32, n0 = p.n0 + j * 32;
            float v[4][4];
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                value(i, j, q, m0 + (p.lane & 31), n0 + q * 8 + (p.lane >> 5) * 4, v[q]);
                Block::put(p.lds, p.lane, 0, q, v[q]);
            }
            // (16 bytes hold the hi or the lo of eight columns)
            Block::each(p.lds, p.lane, [&](int row, int at, u32x4 x) {
                if (m0 + row < p.M && n0 + at / 32 * 8 < Np) *(u32x4 *)(out + (m0 + row) * ld + n0 * 4 + at) = x;
            });
            if (p.tm == p.tn) continue;
#pragma unroll
            for (int q = 0; q < 4; ++q) Block::put_mirrored(p.lds, p.lane, q, v[q]);
            Block::each(p.lds, p.lane, [&](int row, int at, u32x4 x) {
                if (n0 + row < p.N && m0 + at / 32 * 8 < Np) *(u32x4 *)(out + (n0 + row) * ld + m0 * 4 + at) = x;
            });
        }
}

template <int MI, int NI> __device__ __forceinline__ void Gram::run(const Params &e, const f32x16 (&acc)[MI][NI], const Place &p)
{
    const float take = ldexpf(kTake, -2 * e.lift[p.batch]);
    store_symmetric_part<MI, NI>(e.out + p.batch * e.stride, e.ld, p, [&](int i, int j, int q, int, int, float (&v)[4]) {
#pragma unroll
        for (int k = 0; k < 4; ++k) v[k] = acc[i][j][q * 4 + k] * take;
    });
}

template <int MI, int NI> __device__ __forceinline__ void Poly::run(const Params &e, const f32x16 (&acc)[MI][NI], const Place &p)
{
    const char *a = e.a + p.batch * e.stride;
    const int Np = (p.N + 7) & ~7;
    store_symmetric_part<MI, NI>(e.out + p.batch * e.stride, e.ld, p, [&](int i, int j, int q, int m, int n, float (&v)[4]) {
        v[0] = v[1] = v[2] = v[3] = 0.f;
        if (m < p.M && n < Np) load_split(a + m * e.ld, n, v);
#pragma unroll
        for (int k = 0; k < 4; ++k)
            v[k] = kB * v[k] + (kC * kTake) * acc[i][j][q * 4 + k] + (m == n + k && m < p.M ? kA * kStore : 0.f);
    });
}

// a slice's part of S, in float, [slice][batch][r][ld]
struct GramPart : Ending {
    static constexpr bool kSymmetric = true;
    struct Params { float *out; int ld, batch; };
    template <int MI, int NI> static __device__ __forceinline__ void run(const Params &e, const f32x16 (&acc)[MI][NI], const Place &p)
    {
        float *out = e.out + ((long)p.slice * e.batch + p.batch) * p.N * e.ld;
        typedef RowBlock<Fmt::kF32, NI> Block;
#pragma unroll
        for (int i = 0; i < MI; ++i) {
#pragma unroll
            for (int j = 0; j < NI; ++j)
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const float v[4] = {acc[i][j][q * 4], acc[i][j][q * 4 + 1], acc[i][j][q * 4 + 2], acc[i][j][q * 4 + 3]};
                    Block::put(p.lds, p.lane, j, q, v);
                }
            const int m0 = p.m0 + i * 32;
            Block::each(p.lds, p.lane, [&](int row, int at, u32x4 x) {
                if (m0 + row < p.M && p.n0 + at / 4 < e.ld) *(u32x4 *)(out + (long)(m0 + row) * e.ld + p.n0 + at / 4) = x;
            });
        }
    }
};
// ... and S from the slices' parts: 32 x 32 of it to a block, of which a thread has four neighbours of a row
__global__ void __launch_bounds__(256) join_gram_kernel(const float *__restrict__ part, int r, int ld, int batches, int slices, int tile,
                                                        char *__restrict__ out, long ld_out, const int *__restrict__ lift)
{
    if (blockIdx.x * 32 / tile < blockIdx.y * 32 / tile) return; // (below the diagonal's tiles: written as the mirror image)
    const bool mirror = blockIdx.x * 32 / tile != blockIdx.y * 32 / tile;
    // neighbouring threads take neighbouring rows, as the mirrored stores want them
    const int m = blockIdx.y * 32 + (threadIdx.x & 31), n = blockIdx.x * 32 + (threadIdx.x >> 5) * 4;
    float v[4] = {0.f, 0.f, 0.f, 0.f};
    if (m < r && n < ld)
        for (int s0 = 0; s0 < slices; s0 += 8) { // eight slices on their way at a time
            f32x4 x[8];
#pragma unroll
            for (int s = 0; s < 8; ++s)
                x[s] = s0 + s < slices ? *(const f32x4 *)(part + (((long)(s0 + s) * batches + blockIdx.z) * r + m) * ld + n) : f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int s = 0; s < 8; ++s)
#pragma unroll
                for (int e = 0; e < 4; ++e) v[e] += x[s][e];
        }
    const float take = ldexpf(kTake, -2 * lift[blockIdx.z]);
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] *= take;
    store_symmetric(out + blockIdx.z * r * ld_out, ld_out, m, n, r, (r + 7) & ~7, mirror, v);
}

// the next X
struct Next : Ending {
    struct Params { char *out; long ld, stride; };
    template <int MI, int NI> static __device__ __forceinline__ void run(const Params &e, const f32x16 (&acc)[MI][NI], const Place &p)
    {
        char *out = e.out + p.batch * e.stride;
        const int Np = (p.N + 7) & ~7;
        typedef RowBlock<Fmt::kSplit, NI> Block;
#pragma unroll
        for (int i = 0; i < MI; ++i) {
#pragma unroll
            for (int j = 0; j < NI; ++j)
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    float v[4];
#pragma unroll
                    for (int k = 0; k < 4; ++k) v[k] = acc[i][j][q * 4 + k] * kTake;
                    Block::put(p.lds, p.lane, j, q, v);
                }
            const int m0 = p.m0 + i * 32;
            Block::each(p.lds, p.lane, [&](int row, int at, u32x4 x) {
                if (m0 + row < p.M && p.n0 + at / 32 * 8 < Np) *(u32x4 *)(out + (m0 + row) * e.ld + p.n0 * 4 + at) = x;
            });
        }
    }
};

// the result, or the weights' update: out = keep * out + scale * acc
template <typename T, bool UPDATE> struct Last : Ending {
    struct Params { T *out; float keep, scale; const int *lift; };
    template <int MI, int NI> static __device__ __forceinline__ void run(const Params &e, const f32x16 (&acc)[MI][NI], const Place &p)
    {
        T *out = e.out + (long)p.batch * p.M * p.N;
        const bool wide = (p.N & 3) == 0; // rows in whole groups of four
        const float scale = ldexpf(e.scale, -e.lift[p.batch]);
        typedef RowBlock<Fmt::kF32, NI> Block;
#pragma unroll
        for (int i = 0; i < MI; ++i) {
            const int m0 = p.m0 + i * 32;
#pragma unroll
            for (int j = 0; j < NI; ++j)
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    float v[4];
#pragma unroll
                    for (int k = 0; k < 4; ++k) v[k] = scale * acc[i][j][q * 4 + k];
                    Block::put(p.lds, p.lane, j, q, v);
                }
            // (float in LDS for both types: four numbers to a lane, neighbouring lanes side by side)
            Block::each(p.lds, p.lane, [&](int row, int at, u32x4 x) {
                const int m = m0 + row, n = p.n0 + at / 4;
                if (m >= p.M || n >= p.N) return;
                T *o = out + (long)m * p.N + n;
                struct alignas(4 * sizeof(T)) Four { T v[4]; } f;
                if (wide) {
                    if (UPDATE) f = *(const Four *)o;
#pragma unroll
                    for (int k = 0; k < 4; ++k)
                        Elem<T>::store(&f.v[k], UPDATE ? e.keep * Elem<T>::load(&f.v[k]) + __uint_as_float(x[k]) : __uint_as_float(x[k]));
                    *(Four *)o = f;
                } else {
#pragma unroll
                    for (int k = 0; k < 4; ++k)
                        if (n + k < p.N) Elem<T>::store(o + k, UPDATE ? e.keep * Elem<T>::load(o + k) + __uint_as_float(x[k]) : __uint_as_float(x[k]));
                }
            });
        }
    }
};

__device__ __forceinline__ double wave_sum(double v)
{
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) v += __shfl_down(v, off, 64);
    return v;
}

// A 4096 x 4096 step of five iterations takes 3.7 ms, 1.37e12 operations of float products: 0.37 PFLOP/s, 83 % of what a third of a large
// half-precision product reaches.  1000 x 2049 has 128 to 512 tiles of 64 to a product, some 15 launches of 14 to 24 us: latency and the
// compute units' fill.  The passes over the matrix (below) move 8 to 12 bytes an element and are 3 % of it.
//
// Momentum, and each block's part of |U|^2 of its matrix (in double: a gradient's scale is anything).
template <typename TG> __global__ void __launch_bounds__(256)
momentum_kernel(const TG *__restrict__ G, float *__restrict__ M, long size, float mu, int nesterov, double *__restrict__ part)
{
    const TG *g = G + blockIdx.y * size;
    float *m = M ? M + blockIdx.y * size : nullptr;
    double s = 0.0;
    const long step = (long)gridDim.x * 1024;
    const bool wide = (size & 3) == 0;
    for (long i = ((long)blockIdx.x * 256 + threadIdx.x) * 4; i < size; i += step) {
        float u[4], mm[4];
        const int n = (int)min(4L, size - i);
        if (wide) {
            struct alignas(4 * sizeof(TG)) Four { TG v[4]; };
            const Four f = *(const Four *)(g + i);
#pragma unroll
            for (int e = 0; e < 4; ++e) u[e] = Elem<TG>::load(&f.v[e]);
            if (m) *(f32x4 *)mm = *(const f32x4 *)(m + i);
        } else {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                u[e] = e < n ? Elem<TG>::load(g + i + e) : 0.f;
                if (m) mm[e] = e < n ? m[i + e] : 0.f;
            }
        }
        if (m) {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                mm[e] = mu * mm[e] + u[e];
                u[e] = nesterov ? u[e] + mu * mm[e] : mm[e];
            }
            if (wide) *(f32x4 *)(m + i) = *(f32x4 *)mm;
            else
                for (int e = 0; e < n; ++e) m[i + e] = mm[e];
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) s += (double)u[e] * u[e];
    }
    __shared__ double red[4];
    s = wave_sum(s);
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = s;
    __syncthreads();
    if (threadIdx.x == 0) part[blockIdx.y * gridDim.x + blockIdx.x] = ((red[0] + red[1]) + red[2]) + red[3];
}

// X_0, split; a thread takes eight neighbours of a row
template <typename TG> __global__ void __launch_bounds__(256)
normalise_kernel(const TG *__restrict__ G, const float *__restrict__ M, int rows, int cols, float mu, int nesterov,
                 const double *__restrict__ part, int nparts, char *__restrict__ X, long ld, int steps, int *__restrict__ lifts)
{
    const int batch = blockIdx.y;
    __shared__ double red[4];
    double s = (int)threadIdx.x < nparts ? part[batch * nparts + threadIdx.x] : 0.0; // nparts <= 256
    s = wave_sum(s);
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = s;
    __syncthreads();
    // (divided in double: a norm that float does not hold, of a gradient that it does, still has a quotient)
    const double norm = sqrt(((red[0] + red[1]) + red[2]) + red[3]);
    const int lift = ns_lift(norm, steps);
    if (blockIdx.x == 0 && threadIdx.x == 0) lifts[batch] = lift;
    const double scale = ldexp((double)kStore, lift) / (norm + (double)kNsEps);
    const long size = (long)rows * cols;
    const TG *g = G + batch * size;
    const float *m = M ? M + batch * size : nullptr;
    const int per_row = (cols + 7) / 8;
    const bool wide = (cols & 3) == 0;
    for (long c = (long)blockIdx.x * 256 + threadIdx.x; c < (long)rows * per_row; c += (long)gridDim.x * 256) {
        const int row = (int)(c / per_row), n = (int)(c - (long)row * per_row) * 8;
        const long at = (long)row * cols + n;
#pragma unroll
        for (int h = 0; h < 8; h += 4) {
            float u[4] = {0.f, 0.f, 0.f, 0.f};
            if (n + h < cols) {
                float mm[4];
                const int left = min(4, cols - n - h);
                if (wide) {
                    struct alignas(4 * sizeof(TG)) Four { TG v[4]; };
                    const Four f = *(const Four *)(g + at + h);
#pragma unroll
                    for (int e = 0; e < 4; ++e) u[e] = Elem<TG>::load(&f.v[e]);
                    if (m) *(f32x4 *)mm = *(const f32x4 *)(m + at + h);
                } else {
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        if (e < left) {
                            u[e] = Elem<TG>::load(g + at + h + e);
                            if (m) mm[e] = m[at + h + e];
                        }
                }
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    if (m && e < left) u[e] = nesterov ? u[e] + mu * mm[e] : mm[e];
                    u[e] = (float)((double)u[e] * scale);
                }
            }
            store_split(X + batch * (long)rows * ld + row * ld, n + h, u);
        }
    }
}

size_t up(size_t n) { return (n + 255) & ~(size_t)255; }

} // namespace

void plan_muon(const MuonGeom &g, MuonPlan *p)
{
    p->narrow = p->fits = plan_muon_narrow(g, &p->np);
    if (p->narrow) {
        p->bytes = p->np.bytes;
        return;
    }
    p->tall = g.rows > g.cols;
    p->r = p->tall ? g.cols : g.rows;
    p->ld_x = (g.cols + 31) / 32 * 128;
    p->ld_a = (p->r + 31) / 32 * 128;
    p->gram = choose(kSplit, p->r, p->r, g.batch, p->tall ? g.rows : g.cols, true, 16);
    p->poly = choose(kSplit, p->r, p->r, g.batch, p->r, true, 1);
    p->apply = choose(kSplit, g.rows, g.cols, g.batch, p->r, false, 1);
    p->fits = fits_grid(p->gram.shape, tiles_of(p->gram.shape, p->r, p->r, true) * p->gram.slices * g.batch) &&
              fits_grid(p->poly.shape, tiles_of(p->poly.shape, p->r, p->r, true) * g.batch) &&
              fits_grid(p->apply.shape, tiles_of(p->apply.shape, g.rows, g.cols, false) * g.batch);
    const long size = g.rows * g.cols;
    p->sum_blocks = (int)(size / 8192 < 1 ? 1 : size / 8192 > kMaxSumBlocks ? kMaxSumBlocks : size / 8192);
    size_t o = 0;
    p->o_sum = o;
    o += up(sizeof(double) * g.batch * p->sum_blocks);
    p->o_lift = o;
    o += up(sizeof(int) * g.batch);
    for (int i = 0; i < 2; ++i) {
        p->o_x[i] = o;
        o += up((size_t)g.batch * g.rows * p->ld_x);
    }
    p->o_a = o;
    o += up((size_t)g.batch * p->r * p->ld_a);
    p->o_b = o;
    o += up((size_t)g.batch * p->r * p->ld_a);
    p->o_part = o;
    if (p->gram.slices > 1) o += up((size_t)p->gram.slices * g.batch * p->r * ((p->r + 3) & ~3L) * 4);
    p->bytes = o;
}

namespace {

template <typename TG>
hipError_t launch_start(const MuonGeom &g, const MuonPlan &p, const TG *G, float *M, float mu, char *ws, hipStream_t st)
{
    double *part = (double *)(ws + p.o_sum);
    hipLaunchKernelGGL(momentum_kernel<TG>, dim3(p.sum_blocks, g.batch), dim3(256), 0, st, G, M, g.rows * g.cols, mu, (int)g.nesterov, part);
    const long chunks = g.rows * ((g.cols + 7) / 8);
    hipLaunchKernelGGL(normalise_kernel<TG>, dim3((unsigned)(chunks > 256 * 2048 ? 2048 : (chunks + 255) / 256), g.batch), dim3(256), 0, st, G, M,
                       (int)g.rows, (int)g.cols, mu, (int)g.nesterov, (const double *)part, p.sum_blocks, ws + p.o_x[0], p.ld_x, g.steps, (int *)(ws + p.o_lift));
    return hipGetLastError();
}

template <class Epi>
hipError_t launch_apply(const MuonGeom &g, const MuonPlan &p, const char *x, const char *b, const typename Epi::Params &e, hipStream_t st)
{
    Params m{};
    m.M = (int)g.rows;
    m.N = (int)g.cols;
    m.K = (int)p.r;
    m.batch = g.batch;
    const long sx = g.rows * p.ld_x, sb = p.r * p.ld_a;
    m.a = p.tall ? x : b;
    m.b = p.tall ? b : x;
    m.lda = p.tall ? p.ld_x : p.ld_a;
    m.ldb = p.tall ? p.ld_a : p.ld_x;
    m.a_batch = p.tall ? sx : sb;
    m.b_batch = p.tall ? sb : sx;
    if (p.tall) return launch<Split, Lay::kAlong, Lay::kAlong, Epi>(m, e, p.apply, st);
    return launch<Split, Lay::kAlong, Lay::kDown, Epi>(m, e, p.apply, st);
}

} // namespace

hipError_t launch_muon(const MuonGeom &g, const MuonPlan &p, const void *G, float *M, void *W, void *O, float momentum, float keep,
                       float lr, void *ws_, hipStream_t st)
{
    if (p.narrow) return launch_muon_narrow(g, p.np, G, M, W, O, momentum, keep, lr, ws_, st);
    char *ws = (char *)ws_;
    hipError_t e = g.grad_dtype == CAC_F32 ? launch_start(g, p, (const float *)G, M, momentum, ws, st)
                                           : launch_start(g, p, (const bf16_t *)G, M, momentum, ws, st);
    if (e != hipSuccess) return e;
    const long sx = g.rows * p.ld_x, sa = p.r * p.ld_a;
    char *a = ws + p.o_a, *b = ws + p.o_b;
    const int *lift = (const int *)(ws + p.o_lift);
    for (int s = 0; s < g.steps; ++s) {
        char *x = ws + p.o_x[s & 1];
        Params m{};
        m.a = m.b = x;
        m.lda = m.ldb = p.ld_x;
        m.a_batch = m.b_batch = sx;
        m.M = m.N = (int)p.r;
        m.K = (int)(p.tall ? g.rows : g.cols);
        m.batch = g.batch;
        if (p.gram.slices == 1) {
            const Gram::Params eg{a, p.ld_a, sa, lift};
            e = p.tall ? launch<Split, Lay::kDown, Lay::kDown, Gram>(m, eg, p.gram, st) : launch<Split, Lay::kAlong, Lay::kAlong, Gram>(m, eg, p.gram, st);
        } else {
            float *part = (float *)(ws + p.o_part);
            const int ld = (int)((p.r + 3) & ~3L);
            const GramPart::Params eg{part, ld, g.batch};
            e = p.tall ? launch<Split, Lay::kDown, Lay::kDown, GramPart>(m, eg, p.gram, st)
                       : launch<Split, Lay::kAlong, Lay::kAlong, GramPart>(m, eg, p.gram, st);
            if (e != hipSuccess) return e;
            hipLaunchKernelGGL(join_gram_kernel, dim3(cdiv(p.r, 32), cdiv(p.r, 32), g.batch), dim3(256), 0, st, (const float *)part, (int)p.r, ld, g.batch,
                               p.gram.slices, kRows[p.gram.shape], a, p.ld_a, lift);
            e = hipGetLastError();
        }
        if (e != hipSuccess) return e;
        m.a = m.b = a;
        m.lda = m.ldb = p.ld_a;
        m.a_batch = m.b_batch = sa;
        m.K = (int)p.r;
        e = launch<Split, Lay::kAlong, Lay::kAlong, Poly>(m, Poly::Params{b, p.ld_a, sa, a}, p.poly, st);
        if (e != hipSuccess) return e;
        if (s + 1 < g.steps) {
            e = launch_apply<Next>(g, p, x, b, Next::Params{ws + p.o_x[(s + 1) & 1], p.ld_x, sx}, st);
        } else if (W) {
            const float scale = -lr * kTake * kTake;
            e = g.dtype == CAC_F32 ? launch_apply<Last<float, true>>(g, p, x, b, {(float *)W, keep, scale, lift}, st)
                                   : launch_apply<Last<bf16_t, true>>(g, p, x, b, {(bf16_t *)W, keep, scale, lift}, st);
        } else {
            e = g.dtype == CAC_F32 ? launch_apply<Last<float, false>>(g, p, x, b, {(float *)O, 0.f, kTake * kTake, lift}, st)
                                   : launch_apply<Last<bf16_t, false>>(g, p, x, b, {(bf16_t *)O, 0.f, kTake * kTake, lift}, st);
        }
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

} // namespace cac
