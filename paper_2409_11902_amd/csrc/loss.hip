// Softmax cross entropy of a linear classifier, z = H W^T + b, over many classes.  Neither pass keeps the logits:
//
//   forward : lse_t = log sum_v exp z_tv from each tile's maximum and sum of a row, loss_t = lse_t - z_t,label
//   backward: the logits once more, piece of the classes by piece, G_tv = q_t (exp(z_tv - lse_t) - [v = label_t]) from them, then
//             dW = c G^T H and dH = c G W; the rows' gradients are c q_t, c the largest of them, so that a mean's are q = 1 exactly
//             and G is rounded once.
//
// Rows that are left out (label equal to ignore_index, or no class) are taken out of H when it is copied into the workspace: no
// product reads them, whatever stands there, and the products get shorter by them.  Few rows, and short forward passes, stay where
// they are: rows that are left out are loaded as zeros.
// Sums are of 32 bits; G is rounded to bfloat16 for bfloat16 operands (its products' operands are), and held as two halves for float
// (each row's beside the row's largest for dH, each class's beside the class's for dW and db), or as floats where there are few rows.  Of up to 32 bfloat16 rows, whose gradients may hang on a single number of G, what the
// rounding took away is kept as 32 further rows of G: a tile has room for 64 rows, so that products of them cost nothing.
#include "mm_core.h"
#include "train_ends.h"

namespace cac {

namespace {

using namespace mm;

// What the operands are, as they lie and as they are multiplied.
template <class B> struct OfBf16 { typedef bf16_t E; typedef B P; static constexpr bool kSplit = false; static constexpr Fmt kG = Fmt::kBf16; }; // (Bf16, Bf16Odd)
struct OfSplit { typedef float E; typedef Split P; static constexpr bool kSplit = true; static constexpr Fmt kG = Fmt::kSplit; };
template <class R> struct OfRaw { typedef float E; typedef R P; static constexpr bool kSplit = false; static constexpr Fmt kG = Fmt::kF32; }; // (Raw, RawOdd)

constexpr float kLog2e = 1.44269504088896340736f;
// G is stored times 2^14 as two halves, |G| <= 1, which keeps its 23 bits down to 2^-16; below that they end at 2^-39.
constexpr int kStoreG = 14;
constexpr int kMaxParts = 1024;    // blocks that look for a matrix's largest number

__device__ __forceinline__ float wave_max(float v)
{
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) v = fmaxf(v, __shfl_xor(v, off, 64));
    return v;
}

// What the passes over compact rows know about them.  With few rows nothing is compacted: row m is row m of H, and what is known
// about it is looked up where the caller has it.
struct Meta {
    bool direct;
    int T;
    Counts counts;
    const float *lse_in, *gloss;
    int *count;       // [0]: rows that count
    int *exps;        // H and W are stored times 2^exps[0] and 2^exps[1] as two halves
    float *c;         // [0]: the largest of the rows' gradients
    int *uneven;      // [0]: some row's gradient is small beside it (row_exp)
    int *row;         // compact row -> row of H
    int *label;
    float *q, *lse;
    float *zlabel;    // forward: the label's logit
    float *top;       // kMaxParts of H, then of W: largest magnitudes

    __device__ __forceinline__ int rows() const { return direct ? T : *count; }
    __device__ __forceinline__ int row_of(int m) const { return direct ? m : row[m]; }
    // of row m: its class, no class (kOut) where it does not count
    __device__ __forceinline__ int label_of(int m) const { return direct ? (counts(m) ? (int)counts.labels[m] : kOut) : label[m]; }
    __device__ __forceinline__ float lse_of(int m) const
    {
        if (!direct) return lse[m];
        const float l = lse_in[m];
        return l == -INFINITY ? INFINITY : l;
    }
    // the largest finite gradient of a row that counts (called by whole waves)
    __device__ __forceinline__ float largest(int lane) const
    {
        if (!direct) return *c;
        float m = 0.f;
        for (int t = lane; t < T; t += 64) {
            const float g = counts(t) ? fabsf(gloss[t]) : 0.f;
            m = g <= 3.4028235e38f ? fmaxf(m, g) : m;
        }
        return wave_max(m);
    }
    __device__ __forceinline__ float q_of(int m, float largest) const { return direct ? (largest > 0.f ? gloss[m] / largest : gloss[m]) : q[m]; }
    static constexpr int kOut = -(1 << 30);
};
constexpr int kFewRows = 64, kFewFloatRows = 128; // (the plan says when)
constexpr int kLoRow = 32;   // the row of G that the first row's rest is, where rests are kept
__host__ __device__ inline size_t up256(size_t n) { return (n + 255) & ~(size_t)255; }
__host__ __device__ inline size_t meta_bytes(long T) { return 256 + up256(2 * kMaxParts * 4) + 5 * up256(4 * (size_t)T); }
inline Meta meta_at(char *p, long T)
{
    Meta m{};
    m.T = (int)T;
    const size_t n = up256(4 * (size_t)T);
    m.count = (int *)p;
    m.exps = (int *)(p + 64);
    m.c = (float *)(p + 128);
    m.uneven = (int *)(p + 192);
    m.top = (float *)(p + 256);
    p += 256 + up256(2 * kMaxParts * 4);
    m.row = (int *)p;
    m.label = (int *)(p + n);
    m.q = (float *)(p + 2 * n);
    m.lse = (float *)(p + 3 * n);
    m.zlabel = (float *)(p + 4 * n);
    return m;
}

__device__ __forceinline__ int wave_add(int v)
{
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) v += __shfl_xor(v, off, 64);
    return v;
}

// A row whose gradient q (over the largest row's) is small has its G as two halves times 2^-row_exp(q) as well, for dH: a row of dH is a sum of
// its own G.  dW and db, whose sums run over the rows, take G as it is formed again then (small_peak).
constexpr float kSmallRow = 0x1p-8f; // (beside q of 1 and with 2^-39 of it lost: 2^-31 of a row's largest)
__device__ __forceinline__ int row_exp(float q)
{
    int e = 0;
    if (q != 0.f && fabsf(q) < kSmallRow) frexpf(q, &e);
    return e;
}

// Largest finite magnitude of H (rows that count) and of W, a part from every block.  Bound by reading: 1531 x 1001 and 50257 x 1001
// float, 207 MB, in 43 us (4.8 TB/s).
__global__ void __launch_bounds__(256) top_kernel(const float *__restrict__ H, long ld_h, long T, const float *__restrict__ W, long ld_w, long V,
                                                  long D, const Counts counts, int blocks_h, float *__restrict__ top, int *__restrict__ uneven)
{
    if (blockIdx.x == 0 && threadIdx.x == 0) *uneven = 0;
    const bool is_h = (int)blockIdx.x < blocks_h;
    const int block = is_h ? blockIdx.x : blockIdx.x - blocks_h, blocks = is_h ? blocks_h : gridDim.x - blocks_h;
    const float *x = is_h ? H : W;
    const long rows = is_h ? T : V, ld = is_h ? ld_h : ld_w;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    float m = 0.f;
    auto see = [&](float x) {
        const float v = fabsf(x);
        m = v <= 3.4028235e38f ? fmaxf(m, v) : m;
    };
    if (!is_h && ld == D) { // dense and all of it: no rows to tell apart
        const long n4 = rows * D / 4, step = (long)blocks * 256;
        for (long i = (long)block * 256 + threadIdx.x; i < n4; i += step * 8) { // eight accesses of 16 bytes on their way at a time
            f32x4 v[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = i + e * step < n4 ? ((const f32x4 *)x)[i + e * step] : f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int e = 0; e < 8; ++e)
#pragma unroll
                for (int k = 0; k < 4; ++k) see(v[e][k]);
        }
        if (block == 0 && (long)threadIdx.x < rows * D - n4 * 4) see(x[n4 * 4 + threadIdx.x]);
    } else {
        for (long r = (long)block * 4 + wave; r < rows; r += blocks * 4) {
            if (is_h && !counts((int)r)) continue;
            const float *p = x + r * ld;
            long d = lane;
            if ((((uintptr_t)x & 15) | (ld & 3)) == 0) {
                for (d = lane * 4; d + 3 < D; d += 2048) {
                    f32x4 v[8];
#pragma unroll
                    for (int e = 0; e < 8; ++e) v[e] = d + e * 256 + 3 < D ? *(const f32x4 *)(p + d + e * 256) : f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                    for (int e = 0; e < 8; ++e)
#pragma unroll
                        for (int k = 0; k < 4; ++k) see(v[e][k]);
                }
                d = (D & ~3L) + lane;
            }
            for (; d < D; d += 512) {
                float v[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) v[e] = d + e * 64 < D ? p[d + e * 64] : 0.f;
#pragma unroll
                for (int e = 0; e < 8; ++e) see(v[e]);
            }
        }
    }
    __shared__ float red[4];
    m = wave_max(m);
    if (lane == 0) red[wave] = m;
    __syncthreads();
    if (threadIdx.x == 0) top[(is_h ? 0 : kMaxParts) + block] = fmaxf(fmaxf(red[0], red[1]), fmaxf(red[2], red[3]));
}

// The power of two that a matrix is stored times, from its blocks' parts: its largest number becomes one below 2^14.  (Every thread of
// a wave calls, and gets it.)
__device__ __forceinline__ int stored_exp(const float *__restrict__ top, int parts)
{
    float m = 0.f, v[kMaxParts / 64];
#pragma unroll
    for (int k = 0; k < kMaxParts / 64; ++k) { // (all on their way at once)
        const int i = k * 64 + (threadIdx.x & 63);
        v[k] = i < parts ? top[i] : 0.f;
    }
#pragma unroll
    for (int k = 0; k < kMaxParts / 64; ++k) m = fmaxf(m, v[k]);
    m = wave_max(m);
    if (!(m > 0.f)) return 0;
    int e;
    frexpf(m, &e); // m < 2^e
    return min(14 - e, 120);
}

struct PackRows {
    const void *H, *W;
    long ld_h, ld_w;
    int T, D;
    int rows_per_block, row_blocks; // the blocks behind the row blocks pack weights
    int classes;                    // of the weights, from W on
    char *out_w;
    uint32_t *peak;                 // backward: of the classes, to be cleared
    int parts_h, parts_w;  // of the largest magnitudes (float)
    char *out;
    long row_bytes;
    Meta meta;
    // forward: rows that are left out get zeros here
    float *loss, *lse_out;
    // backward
    const float *lse, *gloss;
    void *dH;
};

// 512 numbers of a row of memory from n0 on in float, eight neighbours to a lane, zeros past the row's end.  A row that does not start
// on 16 bytes is read side by side and dealt out through the wave's 2304 bytes of LDS.
constexpr int kShortRow = 128;
constexpr int kDeal = 576; // 512 floats, and 4 after every 32, which keeps the lanes' eights apart
template <typename T> __device__ __forceinline__ void load8(const T *p, int n0, int D, bool aligned, int lane, float *deal, float (&v)[8])
{
    const int n = n0 + lane * 8;
    if (aligned) {
        struct alignas(16) Some { T v[16 / sizeof(T)]; };
        if (n + 8 <= D) {
#pragma unroll
            for (int h = 0; h < (int)sizeof(T) / 2; ++h) {
                const Some s = *(const Some *)(p + n + h * (16 / sizeof(T)));
#pragma unroll
                for (int e = 0; e < (int)(16 / sizeof(T)); ++e) v[h * (16 / sizeof(T)) + e] = Elem<T>::load(&s.v[e]);
            }
            return;
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = n + e < D ? Elem<T>::load(p + n + e) : 0.f;
        return;
    }
    float x[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = n0 + e * 64 + lane < D ? Elem<T>::load(p + n0 + e * 64 + lane) : 0.f;
#pragma unroll
    for (int e = 0; e < 8; ++e) deal[e * 72 + lane + lane / 32 * 4] = x[e];
    asm volatile("" ::: "memory"); // (a wave's LDS accesses are in order; other lanes' stores are read here)
    __builtin_amdgcn_wave_barrier();
    const float *d = deal + lane * 8 + lane / 4 * 4;
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = d[e];
    asm volatile("" ::: "memory");
    __builtin_amdgcn_wave_barrier();
}
// ... and into a packed row (as they are, or two halves times `scale`)
template <class K> __device__ __forceinline__ void store8(char *row, int n, const float (&v)[8], float scale)
{
    if (!K::kSplit) {
        u32x4 u;
#pragma unroll
        for (int e = 0; e < 4; ++e) u[e] = f32x2_to_bf16x2(v[2 * e], v[2 * e + 1]);
        *(u32x4 *)(row + n * 2) = u;
        return;
    }
#pragma unroll
    for (int h = 0; h < 8; h += 4) {
        const float x[4] = {v[h] * scale, v[h + 1] * scale, v[h + 2] * scale, v[h + 3] * scale};
        store_split(row, n + h, x);
    }
}

// Rows that count, one behind the other, and what is known about them.  A block takes a run of rows; where they go follows from the
// labels before them.  With the weights (below) 1531 x 1001 and 50257 x 1001 float in 78 us, 414 MB in and out (5.3 TB/s).
template <class K> __device__ __forceinline__ void pack_rows(const PackRows &p, float *deal)
{
    typedef typename K::E T;
    const Counts &counts = p.meta.counts;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int first = blockIdx.x * p.rows_per_block, last = min(p.T, first + p.rows_per_block);
    __shared__ int red_n[4];
    __shared__ float red_c[4];
    int before = 0;
    float c = 0.f;
    for (int t = threadIdx.x; t < (p.gloss ? p.T : first); t += 256) {
        const bool in = counts(t);
        if (t < first) before += in;
        if (p.gloss && in) {
            const float g = fabsf(p.gloss[t]); // (an infinite or undefined one spoils its own row alone)
            c = g <= 3.4028235e38f ? fmaxf(c, g) : c;
        }
    }
    before = wave_add(before);
    c = wave_max(c);
    if (lane == 0) {
        red_n[wave] = before;
        red_c[wave] = c;
    }
    __syncthreads();
    before = red_n[0] + red_n[1] + red_n[2] + red_n[3];
    c = fmaxf(fmaxf(red_c[0], red_c[1]), fmaxf(red_c[2], red_c[3]));
    const int exp_h = K::kSplit ? stored_exp(p.meta.top, p.parts_h) : 0;
    const float scale = ldexpf(1.f, exp_h);
    if (blockIdx.x == 0 && wave == 0) {
        const int exp_w = K::kSplit ? stored_exp(p.meta.top + kMaxParts, p.parts_w) : 0;
        if (lane == 0) {
            p.meta.exps[0] = exp_h;
            p.meta.exps[1] = exp_w;
            *p.meta.c = c;
        }
    }
    const bool aligned = ((uintptr_t)p.H & 15) == 0 && (p.ld_h * sizeof(T)) % 16 == 0;
    // the waves take turns over the block's rows; 64 rows' labels at a time give every wave the places
    int place = before;
    for (int r0 = first; r0 < last; r0 += 64) {
        const int t = r0 + lane;
        const bool in = t < last && counts(t);
        const uint64_t mask = __ballot(in);
        const int j = place + __popcll(mask & (((uint64_t)1 << lane) - 1));
        if (wave == 0 && t < last) {
            if (in) {
                p.meta.row[j] = t;
                p.meta.label[j] = (int)counts.labels[t];
                if (p.gloss) {
                    const float l = p.lse[t];
                    const float q = c > 0.f ? p.gloss[t] / c : p.gloss[t];
                    p.meta.q[j] = q;
                    if (K::kSplit && row_exp(q) != 0) *p.meta.uneven = 1;
                    // a row whose classes are all masked has no distribution: its probabilities are zeros
                    p.meta.lse[j] = l == -INFINITY ? INFINITY : l;
                }
            } else if (p.loss) {
                p.loss[t] = 0.f;
                p.lse_out[t] = 0.f;
            }
        }
        for (int k = wave; k < min(64, last - r0); k += 4) {
            const int row = r0 + k;
            if (mask >> k & 1) {
                const int jj = p.meta.direct ? row : place + __popcll(mask & (((uint64_t)1 << k) - 1));
                const T *h = (const T *)p.H + (long)row * p.ld_h;
                char *o = p.out + (long)jj * p.row_bytes;
                for (int n0 = 0; n0 < p.D; n0 += 512) {
                    float v[8];
                    load8(h, n0, p.D, aligned, lane, deal, v);
                    if (n0 + lane * 8 < p.D) store8<K>(o, n0 + lane * 8, v, scale);
                }
            } else if (p.dH) {
                T *o = (T *)p.dH + (long)row * p.D;
                for (int n = lane; n < p.D; n += 64) Elem<T>::store(o + n, 0.f);
            }
        }
        place += __popcll(mask);
    }
    if (last == p.T && threadIdx.x == 0) *p.meta.count = place;
}

// A piece of the weights, its rows padded to whole chunks.
template <class K> __device__ __forceinline__ void pack_weights(const PackRows &p, float *deal)
{
    typedef typename K::E T;
    const float s = K::kSplit ? ldexpf(1.f, stored_exp(p.meta.top + kMaxParts, p.parts_w)) : 1.f;
    const bool aligned = ((uintptr_t)p.W & 15) == 0 && (p.ld_w * sizeof(T)) % 16 == 0;
    const int lane = threadIdx.x & 63, rows = 4 * (gridDim.x - p.row_blocks);
    if (K::kSplit && p.peak)
        for (int c = (blockIdx.x - p.row_blocks) * 256 + threadIdx.x; c < p.classes; c += rows * 64) p.peak[c] = 0u;
    // Short rows: a thread to eight numbers, wherever they are (100 x 100 x 60000 float forward: 53 us with a wave to a row, 43 so;
    // of 16 x 252 x 60000 bfloat16 40 and 43).
    if (p.D <= kShortRow) {
        const unsigned per_row = (p.D + 7) / 8, all = p.classes * per_row; // (2^24 at most)
        for (unsigned c = (blockIdx.x - p.row_blocks) * 256 + threadIdx.x; c < all; c += rows * 64) {
            const unsigned row = c / per_row;
            const int n = (c - row * per_row) * 8;
            const T *w = (const T *)p.W + row * p.ld_w + n;
            float v[8];
            if (aligned && n + 8 <= p.D) {
                struct alignas(16) Some { T v[16 / sizeof(T)]; };
#pragma unroll
                for (int h = 0; h < (int)sizeof(T) / 2; ++h) {
                    const Some x = *(const Some *)(w + h * (16 / sizeof(T)));
#pragma unroll
                    for (int e = 0; e < (int)(16 / sizeof(T)); ++e) v[h * (16 / sizeof(T)) + e] = Elem<T>::load(&x.v[e]);
                }
            } else {
#pragma unroll
                for (int e = 0; e < 8; ++e) v[e] = n + e < p.D ? Elem<T>::load(w + e) : 0.f;
            }
            store8<K>(p.out_w + row * p.row_bytes, n, v, s);
        }
        return;
    }
    // a wave to a row
    for (int row = 4 * (blockIdx.x - p.row_blocks) + (threadIdx.x >> 6); row < p.classes; row += rows) {
        const T *w = (const T *)p.W + row * p.ld_w;
        char *out = p.out_w + row * p.row_bytes;
        for (int n0 = 0; n0 < p.D; n0 += 512) {
            float v[8];
            load8(w, n0, p.D, aligned, lane, deal, v);
            if (n0 + lane * 8 < p.D) store8<K>(out, n0 + lane * 8, v, s);
        }
    }
}
template <class K> __global__ void __launch_bounds__(256) pack_kernel(const PackRows p)
{
    __shared__ float deal[4][kDeal];
    if ((int)blockIdx.x < p.row_blocks) pack_rows<K>(p, deal[threadIdx.x >> 6]);
    else pack_weights<K>(p, deal[threadIdx.x >> 6]);
}

// four neighbours of b from n on, zeros past its end
template <typename T> __device__ __forceinline__ void load_bias(const T *b, int n, int N, float (&v)[4])
{
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = b && n + e < N ? Elem<T>::load(b + n + e) : 0.f;
}

// ---- endings of the products
// forward: maximum and sum of exp of a row over a wave's columns, and the label's logit
template <class K> struct Stats : Ending {
    typedef typename K::E T;
    static constexpr bool kCountsM = true;
    struct Params {
        const T *b;
        Meta meta;
        float *part;      // [2 * parts][T]
        long T_rows;
        int part0, v0;    // the piece's first part, its first class
    };
    template <int MI, int NI> static __device__ __forceinline__ void run(const Params &e, const f32x16 (&acc)[MI][NI], const Place &p)
    {
        const int ze = K::kSplit ? -(e.meta.exps[0] + e.meta.exps[1]) : 0;
        const int part = e.part0 + p.part;
#pragma unroll
        for (int i = 0; i < MI; ++i) {
            const int m = p.m0 + i * 32 + (p.lane & 31);
            const int label = m < p.M ? e.meta.label_of(m) - e.v0 : Meta::kOut;
            float top = -INFINITY, sum = 0.f, z[NI][16];
#pragma unroll
            for (int j = 0; j < NI; ++j)
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const int n = p.n0 + j * 32 + q * 8 + (p.lane >> 5) * 4;
                    float bias[4];
                    load_bias(e.b, n, p.N, bias);
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        const float v = (K::kSplit ? ldexpf(acc[i][j][q * 4 + k], ze) : acc[i][j][q * 4 + k]) + bias[k];
                        z[j][q * 4 + k] = n + k < p.N ? v : -INFINITY;
                        if (n + k == label && n + k < p.N) e.meta.zlabel[m] = v;
                        top = fmaxf(top, z[j][q * 4 + k]);
                    }
                }
            top = fmaxf(top, __shfl_xor(top, 32, 64));
            const float shift = top == -INFINITY ? 0.f : top;
#pragma unroll
            for (int j = 0; j < NI; ++j)
#pragma unroll
                for (int k = 0; k < 16; ++k) sum += __builtin_amdgcn_exp2f((z[j][k] - shift) * kLog2e);
            sum += __shfl_xor(sum, 32, 64);
            if (p.lane < 32 && m < p.M) {
                e.part[(2L * part) * e.T_rows + m] = top;
                e.part[(2L * part + 1) * e.T_rows + m] = sum;
            }
        }
    }
};

// lse and loss of a compact row from its parts: ROWS rows to a block, 256 / ROWS threads to a row.  4096 rows of 500 parts in 8 us.
template <int ROWS> __global__ void __launch_bounds__(256) join_kernel(const Meta meta, const float *__restrict__ part, int parts, long T_rows,
                                                                       float *__restrict__ loss, float *__restrict__ lse)
{
    constexpr int kThreads = 256 / ROWS;
    const int count = meta.rows();
    const int r = threadIdx.x % ROWS, s = threadIdx.x / ROWS;
    const int j = blockIdx.x * ROWS + r;
    float top = -INFINITY, sum = 0.f;
    if (j < count)
        for (int k0 = s; k0 < parts; k0 += 8 * kThreads) { // eight parts on their way at a time
            float t[8], u[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const int k = k0 + e * kThreads;
                t[e] = k < parts ? part[2L * k * T_rows + j] : -INFINITY;
                u[e] = k < parts ? part[(2L * k + 1) * T_rows + j] : 0.f;
            }
            float m = top;
#pragma unroll
            for (int e = 0; e < 8; ++e) m = fmaxf(m, t[e]);
            const float shift = m == -INFINITY ? 0.f : m;
            sum *= __builtin_amdgcn_exp2f((top - shift) * kLog2e);
#pragma unroll
            for (int e = 0; e < 8; ++e) sum += u[e] * __builtin_amdgcn_exp2f((t[e] - shift) * kLog2e);
            top = m;
        }
    // the threads of a row, in halves
    __shared__ float tops[256], sums[256];
    tops[threadIdx.x] = top;
    sums[threadIdx.x] = sum;
    __syncthreads();
#pragma unroll
    for (int n = kThreads / 2; n > 0; n >>= 1) {
        if (s < n) {
            const int other = threadIdx.x + n * ROWS;
            const float m = fmaxf(tops[threadIdx.x], tops[other]), shift = m == -INFINITY ? 0.f : m;
            sums[threadIdx.x] = sums[threadIdx.x] * __builtin_amdgcn_exp2f((tops[threadIdx.x] - shift) * kLog2e) +
                                sums[other] * __builtin_amdgcn_exp2f((tops[other] - shift) * kLog2e);
            tops[threadIdx.x] = m;
        }
        __syncthreads();
    }
    if (s == 0 && j < count) {
        const float l = tops[r] + logf(sums[r]);
        const int t = meta.row_of(j);
        if (meta.label_of(j) == Meta::kOut) {
            loss[t] = lse[t] = 0.f;
        } else {
            const float z = meta.zlabel[j];
            lse[t] = l;
            loss[t] = z == -INFINITY ? INFINITY : l - z; // (a masked label's loss, also where every class is masked)
        }
    }
}

// four neighbours of a row of G
template <class K> __device__ __forceinline__ void store_gradient(char *row, int n, const float (&g)[4])
{
    if (K::kG == Fmt::kSplit) {
        const float v[4] = {g[0] * (float)(1 << kStoreG), g[1] * (float)(1 << kStoreG), g[2] * (float)(1 << kStoreG), g[3] * (float)(1 << kStoreG)};
        store_split(row, n, v);
    } else if (K::kG == Fmt::kF32) {
        *(f32x4 *)(row + n * 4) = f32x4{g[0], g[1], g[2], g[3]};
    } else {
        u32x2 u;
        u[0] = f32x2_to_bf16x2(g[0], g[1]);
        u[1] = f32x2_to_bf16x2(g[2], g[3]);
        *(u32x2 *)(row + n * 2) = u;
    }
}

// what rounding to bfloat16 takes away
__device__ __forceinline__ float rest_of(float g)
{
    const float r = g - bf16_to_f32(f32_to_bf16(g));
    return g - g == 0.f ? r : 0.f; // (an infinite or undefined one has none)
}

// ---- Classes that no row thinks probable.  dW and db of a class are sums of its own G, so what 2^-39 of the largest G does not hold would
// be all of a class whose G lies down there.  The pass that forms G as two halves leaves every class's largest |G|; where that is below 2^-16, the
// class's G is formed once more, times a power of two of its own, for dW and db (dH has G as it was first: there a row's G are added
// up, improbable beside probable ones).  So is all of G where rows' gradients differ much (row_exp).  Tiles without such a class end at once.  Both passes of 512 x 512 x 1500 and 1000 x 1001 x 50257:
// 52 and 1600 us without all this, 55 and 1620 where no class is improbable, 62 and 1920 where all tiles are formed again.
constexpr float kSmallPeak = 0x1p-16f;
__device__ __forceinline__ bool small_peak(uint32_t peak)
{
    const float m = __uint_as_float(peak);
    return m > 0.f && m < kSmallPeak;
}
// a class's G are below 2^peak_exp (and stored times 2^-peak_exp)
__device__ __forceinline__ int peak_exp(uint32_t peak)
{
    int e = 0;
    if (small_peak(peak)) frexpf(__uint_as_float(peak), &e);
    return e;
}
// Whether G of `count` classes is formed again: 1 or 0, asked by a whole wave.  (A number, which the compiler has to have: where this was a
// condition of branches it left out the one that chooses between two places of G.)
__device__ __forceinline__ int formed_again(const Meta &meta, const uint32_t *peak, int first, int count, int lane)
{
    int any = *meta.uneven;
    for (int k = lane; k < count; k += 64) any |= small_peak(peak[first + k]);
    return __builtin_amdgcn_readfirstlane(__ballot(any != 0) != 0);
}
// `again` where r is 1, else `a`
__device__ __forceinline__ const char *either(const void *a, const char *again, int r)
{
    const uint64_t x = (uint64_t)(uintptr_t)a, at = x ^ ((x ^ (uint64_t)(uintptr_t)again) & -(uint64_t)r);
    const uint32_t lo = __builtin_amdgcn_readfirstlane((uint32_t)at), hi = __builtin_amdgcn_readfirstlane((uint32_t)(at >> 32));
    return (const char *)(uintptr_t)((uint64_t)hi << 32 | lo);
}
// (numbers are not negative, so that they are ordered as their bits are; the largest does not depend on the order of arrival)
__device__ __forceinline__ void raise_peak(uint32_t *peak, float v) { atomicMax(peak, __float_as_uint(v)); }
// of 2 N numbers N to a lane, the larger of its own and of the lane's 2 N apart
template <int N> __device__ __forceinline__ void share_out(float (&v)[16], int lane)
{
    const bool up = lane & 2 * N;
#pragma unroll
    for (int k = 0; k < N; ++k) v[k] = fmaxf(up ? v[k + N] : v[k], __shfl_xor(up ? v[k] : v[k + N], 2 * N, 64));
}
// of a wave's 32 NI columns: v[j][4 q + k] as C lies, largest of the wave's blocks of rows.  Lanes that hold rows of the same columns share the numbers out.
template <int NI> __device__ __forceinline__ void raise_peaks(uint32_t *peak, float (&v)[NI][16], const Place &p)
{
#pragma unroll
    for (int j = 0; j < NI; ++j) {
        share_out<8>(v[j], p.lane);
        share_out<4>(v[j], p.lane);
        share_out<2>(v[j], p.lane);
        share_out<1>(v[j], p.lane);
        const float top = fmaxf(v[j][0], __shfl_xor(v[j][0], 1, 64));
        const int at = p.lane >> 1 & 15, n = p.n0 + j * 32 + (at >> 2) * 8 + (p.lane >> 5) * 4 + (at & 3);
        if (!(p.lane & 1) && n < p.N) raise_peak(peak + n, top);
    }
}

// backward: G of a piece.  AGAIN: of two halves, of tiles with a class whose G are small, every class times its power of two.
template <class K, bool AGAIN = false> struct Grad : Ending {
    typedef typename K::E T;
    static constexpr bool kCountsM = true, kGated = AGAIN;
    struct Params {
        const T *b;
        Meta meta;
        char *out;
        long ld;
        int v0;
        bool rests;
        uint32_t *peak;   // of two halves: [classes], raised (AGAIN: read)
    };
    static __device__ __forceinline__ bool wanted(const Params &e, int first, int count, int lane)
    {
        return formed_again(e.meta, e.peak, first, count, lane) != 0;
    }
    template <int MI, int NI> static __device__ __forceinline__ void run(const Params &e, const f32x16 (&acc)[MI][NI], const Place &p)
    {
        const int ze = K::kSplit ? -(e.meta.exps[0] + e.meta.exps[1]) : 0;
        const float largest = e.meta.largest(p.lane);
        const int Np = (p.N + 7) & ~7;
        typedef RowBlock<K::kG, NI> Block;
        constexpr int kIn16 = sizeof(T) == 4 ? 32 : 16; // bytes that eight columns take
        constexpr bool kPeaks = K::kSplit && !AGAIN;
        float peaks[kPeaks ? NI : 1][16] = {};
#pragma unroll
        for (int i = 0; i < MI; ++i) {
            const int m0 = p.m0 + i * 32, m = min(m0 + (p.lane & 31), p.M - 1);
            const int label = e.meta.label_of(m) - e.v0;
            const bool in = label > Meta::kOut / 2;
            const float q_row = e.meta.q_of(m, largest), lse = e.meta.lse_of(m);
            const int q_exp = kPeaks ? row_exp(q_row) : 0;
            const float q_stored = kPeaks ? ldexpf(q_row, kStoreG - q_exp) : q_row;
            constexpr bool kRests = K::kG == Fmt::kBf16 && MI * NI == 1; // (few rows take the smallest tiles)
            float kept[kRests ? 16 : 1];
#pragma unroll
            for (int j = 0; j < NI; ++j)
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const int n = p.n0 + j * 32 + q * 8 + (p.lane >> 5) * 4;
                    float bias[4], g[4];
                    load_bias(e.b, n, p.N, bias);
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        const float z = (K::kSplit ? ldexpf(acc[i][j][q * 4 + k], ze) : acc[i][j][q * 4 + k]) + bias[k];
                        const float x = __builtin_amdgcn_exp2f((z - lse) * kLog2e) - (n + k == label ? 1.f : 0.f);
                        const float stored = AGAIN ? ldexpf(q_row * x, kStoreG - peak_exp(e.peak[min(n + k, p.N - 1)])) : q_stored * x;
                        g[k] = n + k < p.N && in ? stored : 0.f;
                        if constexpr (kPeaks) peaks[j][q * 4 + k] = fmaxf(peaks[j][q * 4 + k], fabsf(q_row * x));
                        if constexpr (kRests) kept[q * 4 + k] = g[k];
                    }
                    Block::put(p.lds, p.lane, j, q, g);
                }
            auto store = [&](char *out) {
                Block::each(p.lds, p.lane, [&](int row, int at, u32x4 x) {
                    if (m0 + row < p.M && p.n0 + at / kIn16 * 8 < Np) *(u32x4 *)(out + (long)(m0 + row) * e.ld + p.n0 / 8 * kIn16 + at) = x;
                });
            };
            store(e.out);
            if constexpr (kRests) {
                if (!e.rests) continue;
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const float r[4] = {rest_of(kept[q * 4]), rest_of(kept[q * 4 + 1]), rest_of(kept[q * 4 + 2]), rest_of(kept[q * 4 + 3])};
                    Block::put(p.lds, p.lane, 0, q, r);
                }
                store(e.out + kLoRow * e.ld);
            }
        }
        if constexpr (kPeaks) raise_peaks<NI>(e.peak, peaks, p);
    }
};

template <typename T> __device__ __forceinline__ void store_four(T *o, int n, int N, bool wide, const float (&v)[4])
{
    if (wide) {
        struct alignas(4 * sizeof(T)) Four { T v[4]; } f;
#pragma unroll
        for (int k = 0; k < 4; ++k) Elem<T>::store(&f.v[k], v[k]);
        *(Four *)o = f;
        return;
    }
#pragma unroll
    for (int k = 0; k < 4; ++k)
        if (n + k < N) Elem<T>::store(o + k, v[k]);
}

// What a product is multiplied by on its way out: a float, and of two halves a power of two beside it (one float would have to hold what the
// operands were stored times, which the product still is: results that float holds would meet a factor that it does not).
template <bool SPLIT> struct Factor {
    float f;
    int e;
    __device__ __forceinline__ Factor(float largest, int exponent) : f(largest), e(0)
    {
        if (SPLIT) {
            f = frexpf(largest, &e);
            e += exponent;
        }
    }
    __device__ __forceinline__ float operator()(float v) const { return SPLIT ? ldexpf(f * v, e) : f * v; }
};

// 32 rows of a product, times s, into a wave's LDS; zeros where the lane's row is left out
template <class S, int MI, int NI> __device__ __forceinline__ void put_scaled(const f32x16 (&acc)[MI][NI], int i, S s, const Place &p, bool out = false)
{
#pragma unroll
    for (int j = 0; j < NI; ++j)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            float v[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) v[k] = out ? 0.f : s(acc[i][j][q * 4 + k]);
            RowBlock<Fmt::kF32, NI>::put(p.lds, p.lane, j, q, v);
        }
}

// dW of a piece
template <class K> struct OutW : Ending {
    typedef typename K::E T;
    static constexpr bool kOther = K::kSplit;
    struct Params {
        T *out;
        Meta meta;
        const uint32_t *peak; // of two halves, and where G lies that was formed again, if it is elsewhere
        const char *again;
    };
    static __device__ __forceinline__ const void *operand_a(const Params &e, const void *a, int first, int count, int lane)
    {
        return e.again ? either(a, e.again, formed_again(e.meta, e.peak, first, count, lane)) : a;
    }
    template <int MI, int NI> static __device__ __forceinline__ void run(const Params &e, const f32x16 (&acc)[MI][NI], const Place &p)
    {
        const Factor<K::kSplit> s(e.meta.largest(p.lane), K::kSplit ? -kStoreG - e.meta.exps[0] : 0);
        typedef RowBlock<Fmt::kF32, NI> Block;
        const bool wide = (p.N & 3) == 0;
#pragma unroll
        for (int i = 0; i < MI; ++i) {
            const int m0 = p.m0 + i * 32;
            Factor<K::kSplit> of_class = s;
            if (K::kSplit) of_class.e += peak_exp(e.peak[min(m0 + (p.lane & 31), p.M - 1)]);
            put_scaled(acc, i, of_class, p);
            Block::each(p.lds, p.lane, [&](int row, int at, u32x4 x) {
                const int m = m0 + row, n = p.n0 + at / 4;
                if (m < p.M && n < p.N) store_four(e.out + (long)m * p.N + n, n, p.N, wide, {__uint_as_float(x[0]), __uint_as_float(x[1]), __uint_as_float(x[2]), __uint_as_float(x[3])});
            });
        }
    }
};

// dH: the result, or sums of a slice (added to what the pieces before left)
template <class K> struct OutH : Ending {
    typedef typename K::E T;
    struct Params { T *out; float *sums; long slice_stride; int add; bool rests; Meta meta; };
    template <int MI, int NI> static __device__ __forceinline__ void run(const Params &e, const f32x16 (&acc)[MI][NI], const Place &p)
    {
        const Factor<K::kSplit> s(e.meta.largest(p.lane), K::kSplit ? -kStoreG - e.meta.exps[1] : 0);
        typedef RowBlock<Fmt::kF32, NI> Block;
        const bool wide = (p.N & 3) == 0;
#pragma unroll
        for (int i = 0; i < MI; ++i) {
            const int m0 = p.m0 + i * 32;
            const bool rests = K::kG == Fmt::kBf16 && e.rests; // (32 rows and their rests: neighbouring waves of one tile)
            // a row that is left out has zeros in G where nothing is compacted, and a zero times an infinite weight is none
            const int m = m0 + (p.lane & 31), row = rests && m >= kLoRow ? m - kLoRow : m;
            Factor<K::kSplit> of_row = s;
            if (K::kSplit) of_row.e += row_exp(e.meta.q[min(m, p.M - 1)]);
            put_scaled(acc, i, of_row, p, e.meta.direct && row < e.meta.T && e.meta.label_of(row) == Meta::kOut);
            if (rests) {
                __syncthreads();
                if (m0 >= kLoRow) return;
            }
            Block::each(p.lds, p.lane, [&](int row, int at, u32x4 x) {
                const int m = m0 + row, n = p.n0 + at / 4;
                if (m >= (rests ? e.meta.T : p.M) || n >= p.N) return;
                float v[4] = {__uint_as_float(x[0]), __uint_as_float(x[1]), __uint_as_float(x[2]), __uint_as_float(x[3])};
                if (rests) {
                    const f32x4 r = *(const f32x4 *)(p.lds + p.lds_rows + row * Block::kPitch + at);
#pragma unroll
                    for (int k = 0; k < 4; ++k) v[k] += r[k];
                }
                if (!e.sums) {
                    store_four(e.out + (long)e.meta.row_of(m) * p.N + n, n, p.N, wide, v);
                    return;
                }
                float *o = e.sums + p.slice * e.slice_stride + (long)m * p.N + n;
                if (e.add) {
                    if (wide) {
                        const f32x4 old = *(const f32x4 *)o;
#pragma unroll
                        for (int k = 0; k < 4; ++k) v[k] += old[k];
                    } else {
#pragma unroll
                        for (int k = 0; k < 4; ++k)
                            if (n + k < p.N) v[k] += o[k];
                    }
                }
                store_four(o, n, p.N, wide, v);
            });
        }
    }
};

// dH from the slices' sums, four numbers of a compact row to a thread.  WAVES: of few slices every thread adds up its own; of many the
// block's waves take turns over them.
template <typename T, bool WAVES> __global__ void __launch_bounds__(256)
finish_rows_kernel(const Meta meta, const float *__restrict__ sums, long slice_stride, int slices, int D, T *__restrict__ dH)
{
    if ((int)blockIdx.x >= meta.rows()) return;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, n = WAVES ? blockIdx.y * 256 + lane * 4 : (int)(blockIdx.y * 1024 + threadIdx.x * 4);
    const long at = (long)blockIdx.x * D + n;
    const bool wide = (D & 3) == 0;
    constexpr int kTurn = WAVES ? 4 : 1;
    float v[4] = {0.f, 0.f, 0.f, 0.f};
    if (n < D)
        for (int s0 = WAVES ? wave : 0; s0 < slices; s0 += 4 * kTurn) { // four slices on their way at a time
            float x[4][4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int s = s0 + e * kTurn;
                const float *p = sums + s * slice_stride + at;
                if (wide) {
                    const f32x4 y = s < slices ? *(const f32x4 *)p : f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                    for (int k = 0; k < 4; ++k) x[e][k] = y[k];
                } else {
#pragma unroll
                    for (int k = 0; k < 4; ++k) x[e][k] = s < slices && n + k < D ? p[k] : 0.f;
                }
            }
#pragma unroll
            for (int e = 0; e < 4; ++e)
#pragma unroll
                for (int k = 0; k < 4; ++k) v[k] += x[e][k];
        }
    if (WAVES) {
        __shared__ f32x4 red[3][64];
        if (wave > 0) red[wave - 1][lane] = f32x4{v[0], v[1], v[2], v[3]};
        __syncthreads();
        if (wave > 0) return;
#pragma unroll
        for (int w = 0; w < 3; ++w)
#pragma unroll
            for (int k = 0; k < 4; ++k) v[k] += red[w][lane][k];
    }
    if (n < D) store_four(dH + (long)meta.row_of(blockIdx.x) * D + n, n, D, wide, v);
}

// db of a piece: the columns' sums of G, eight columns to a thread, the block's four waves over the rows
template <class K> struct Bias {
    typedef typename K::E T;
    Meta meta;
    const char *G;
    long ld;
    int V;
    T *db;
    bool rests;
    const uint32_t *peak; // as OutW's
    const char *again;
};
template <class K> __device__ __forceinline__ void bias_sums(const Bias<K> &p, int block, float (*red)[64])
{
    typedef typename K::E T;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int rows = p.meta.rows(), count = K::kG == Fmt::kBf16 && p.rests ? 2 * rows : rows;
    const float largest = p.meta.largest(lane);
    // 8 chunks of columns by 8 rows to a wave
    const int chunk = block * 8 + (lane & 7), n = chunk * 8;
    const char *G = p.G;
    if (K::kSplit && p.again) G = either(G, p.again, formed_again(p.meta, p.peak, block * 64, min(p.V - block * 64, 64), lane));
    float s[8] = {};
    if (n < p.V)
        for (int m = wave * 8 + (lane >> 3); m < count; m += 32) {
            const char *g = G + (long)(m < rows ? m : m - rows + kLoRow) * p.ld + (long)chunk * (sizeof(T) == 4 ? 32 : 16);
            if (K::kG == Fmt::kF32) {
                const f32x4 lo = *(const f32x4 *)g, hi = *(const f32x4 *)(g + 16);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    s[e] += lo[e];
                    s[e + 4] += hi[e];
                }
            } else if (K::kSplit) {
                const f16x8 hi = *(const f16x8 *)g, lo = *(const f16x8 *)(g + 16);
#pragma unroll
                for (int e = 0; e < 8; ++e) s[e] += (float)hi[e] + (float)lo[e];
            } else {
                struct alignas(16) Eight { bf16_t v[8]; };
                const Eight v = *(const Eight *)g;
#pragma unroll
                for (int e = 0; e < 8; ++e) s[e] += bf16_to_f32(v.v[e]);
            }
        }
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        s[e] += __shfl_xor(s[e], 8, 64);
        s[e] += __shfl_xor(s[e], 16, 64);
        s[e] += __shfl_xor(s[e], 32, 64);
        if (lane < 8) red[wave][lane * 8 + e] = s[e];
    }
    __syncthreads();
    if (threadIdx.x < 64 && block * 64 + (int)threadIdx.x < p.V) {
        const Factor<K::kSplit> c(largest, K::kSplit ? peak_exp(p.peak[block * 64 + threadIdx.x]) - kStoreG : 0);
        Elem<T>::store(p.db + block * 64 + threadIdx.x, c(((red[0][lane] + red[1][lane]) + red[2][lane]) + red[3][lane]));
    }
}
template <class K> __global__ void __launch_bounds__(256) bias_kernel(const Bias<K> p)
{
    __shared__ float red[4][64];
    bias_sums(p, blockIdx.x, red);
}

// dW of few rows: a wave holds G of 32 classes in registers and passes over columns of H, which needs neither LDS nor a meeting; the
// stores of dW are what takes time: with dH, which reads W, 16 x 1024 x 100000 in 162 us of float and 69 of bfloat16 (820 and 410 MB in
// and out, 5.1 and 5.9 TB/s, some of it cached; as tiles of a product 324 and 169).  ROWS: T or more, a power of two.
template <class K> struct Few {
    typedef typename K::E T;
    Meta meta;
    const char *G;
    const T *H;
    long ld_g, ld_h;   // bytes
    int V, D;
    T *out;
    int runs, run;     // runs of columns that D is cut into; blocks of columns in one
};
// Columns of a block: a lane has one of float, two neighbours of bfloat16.
template <class K> constexpr int kFewColumns = sizeof(typename K::E) == 4 ? 32 : 64;
template <class K, int ROWS> __device__ __forceinline__ void few_rows(const Few<K> &p, unsigned block)
{
    typedef typename K::E T;
    constexpr bool kFloat = sizeof(T) == 4;
    constexpr int kHave = ROWS < 32 ? ROWS / 2 : 16; // rows of H that a lane has at a time, and as many under way
    const int lane = threadIdx.x & 63, c = lane & 31, half = lane >> 5;
    const unsigned job = __builtin_amdgcn_readfirstlane(block * 4 + (threadIdx.x >> 6));
    const int v0 = __builtin_amdgcn_readfirstlane(job / p.runs) * 32, first = (int)(job % p.runs) * p.run * kFewColumns<K>;
    if (v0 >= p.V) return;
    const int last = min(p.D, first + p.run * kFewColumns<K>), rows = p.meta.T;
    // the lane's k-th row of H and G: 2 k + half of float, 8 neighbours of every 16 for bfloat16
    constexpr int kHalf = kFloat ? 1 : 8;
    auto row = [&](int k) { return (kFloat ? 2 * k : k / 8 * 16 + k % 8) + half * kHalf; };
    // rows that count, from the lane's first on (64 to a pair of words)
    uint32_t there[4];
    bool whole = true;
#pragma unroll
    for (int w = 0; w < (ROWS > 64 ? 2 : 1); ++w) {
        const uint64_t all = __ballot(w * 64 + lane < rows && p.meta.counts(w * 64 + lane)), mine = all >> (half * kHalf);
        there[2 * w] = (uint32_t)mine;
        there[2 * w + 1] = (uint32_t)(mine >> 32);
        whole = whole && all == ~0ull >> (ROWS < 64 ? 64 - ROWS : 0);
    }
    auto counts = [&](int k) {
        const int b = kFloat ? 2 * k : k / 8 * 16 + k % 8;
        return (there[b / 32] >> b % 32 & 1) != 0;
    };
    const float scale = p.meta.largest(lane);
    const int gv = min(v0 + c, (p.V + 7) / 8 * 8 - 1);
    uint32_t g[kFloat ? ROWS / 2 : ROWS / 4], h[2][kHave];
    constexpr bool kRests = !kFloat && ROWS <= kLoRow;
    uint32_t low[kRests ? ROWS / 4 : 1];
#pragma unroll
    for (int k = 0; k < ROWS / 2; ++k) {
        const char *r = p.G + min(row(k), rows - 1) * p.ld_g;
        if (kFloat) {
            g[k] = ((const uint32_t *)r)[gv];
            g[k] = counts(k) ? g[k] : 0u;
        } else {
            uint32_t v = ((const uint16_t *)r)[gv];
            v = counts(k) ? v : 0u;
            if (k % 2) g[k / 2] |= v << 16;
            else g[k / 2] = v;
            if constexpr (kRests) {
                v = ((const uint16_t *)(r + kLoRow * p.ld_g))[gv];
                v = counts(k) ? v : 0u;
                if (k % 2) low[k / 2] |= v << 16;
                else low[k / 2] = v;
            }
        }
    }
    const uint32_t ld = p.ld_h, end = (rows - 1) * ld; // (bytes: 128 rows are less than 2^32)
    auto read = [&](int b, int n0, int k0) {
        uint32_t mine = row(0) * ld;
        asm volatile("" : "+v"(mine)); // (the rows' places are worked out again: kept they take half of the registers)
        const uint32_t n = min(n0 + c * (kFloat ? 1 : 2), (p.D - 1) & (kFloat ? ~0 : ~1)) * sizeof(T);
#pragma unroll
        for (int k = 0; k < kHave; ++k) {
            const uint32_t r = min(mine + (uint32_t)(row(k0 + k) - row(0)) * ld, end);
            h[b][k] = *(const uint32_t *)((const char *)p.H + (r + n));
        }
    };
    constexpr int kSets = kFloat ? 1 : 2; // (the even and the odd columns of bfloat16)
    f32x16 acc[kSets];
    auto multiply = [&](int b, int k0) {
        if (k0 == 0)
#pragma unroll
            for (int s = 0; s < kSets; ++s)
#pragma unroll
                for (int r = 0; r < 16; ++r) acc[s][r] = 0.f;
        if (!whole) // whatever stands in a row that does not count
#pragma unroll
            for (int k = 0; k < kHave; ++k) h[b][k] = counts(k0 + k) ? h[b][k] : 0u;
        if constexpr (kFloat) {
#pragma unroll
            for (int k = 0; k < kHave; ++k) acc[0] = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(g[k0 + k]), __uint_as_float(h[b][k]), acc[0], 0, 0, 0);
        } else {
#pragma unroll
            for (int k = 0; k < kHave; k += 8) {
                union { uint32_t u[4]; s16x8 v; } a, even, odd;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    a.u[e] = g[(k0 + k) / 2 + e];
                    even.u[e] = __builtin_amdgcn_perm(h[b][k + 2 * e + 1], h[b][k + 2 * e], 0x05040100u);
                    odd.u[e] = __builtin_amdgcn_perm(h[b][k + 2 * e + 1], h[b][k + 2 * e], 0x07060302u);
                }
                acc[0] = product<Bf16>(a.v, even.v, acc[0]);
                acc[kSets - 1] = product<Bf16>(a.v, odd.v, acc[kSets - 1]);
                if constexpr (kRests) {
#pragma unroll
                    for (int e = 0; e < 4; ++e) a.u[e] = low[(k0 + k) / 2 + e];
                    acc[0] = product<Bf16>(a.v, even.v, acc[0]);
                    acc[kSets - 1] = product<Bf16>(a.v, odd.v, acc[kSets - 1]);
                }
            }
        }
    };
    auto write = [&](int n0) {
        const int n = n0 + c * (kFloat ? 1 : 2);
        T *o = p.out + (long)v0 * p.D + n;
        if (n < p.D)
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                const int v = r / 4 * 8 + half * 4 + r % 4;
                if (v0 + v >= p.V) continue;
                if constexpr (kFloat) o[v * p.D] = scale * acc[0][r];
                else if (p.D % 2 == 0) *(uint32_t *)(o + v * p.D) = f32x2_to_bf16x2(scale * acc[0][r], scale * acc[kSets - 1][r]);
                else {
                    o[v * p.D] = f32_to_bf16(scale * acc[0][r]);
                    if (n + 1 < p.D) o[v * p.D + 1] = f32_to_bf16(scale * acc[kSets - 1][r]);
                }
            }
    };
    constexpr int kCols = kFewColumns<K>;
    read(0, first, 0);
    if constexpr (ROWS > 32) {
        constexpr int kTimes = ROWS / 2 / kHave; // (even: a block ends with the registers that it began with)
        for (int n0 = first; n0 < last; n0 += kCols) {
#pragma unroll
            for (int t = 0; t < kTimes; ++t) {
                if (t + 1 < kTimes) read((t + 1) & 1, n0, (t + 1) * kHave);
                else if (n0 + kCols < last) read(0, n0 + kCols, 0);
                multiply(t & 1, t * kHave);
            }
            write(n0);
        }
    } else {
        for (int n0 = first; n0 < last; n0 += 2 * kCols) {
            if (n0 + kCols < last) read(1, n0 + kCols, 0);
            multiply(0, 0);
            write(n0);
            if (n0 + kCols >= last) break;
            if (n0 + 2 * kCols < last) read(0, n0 + 2 * kCols, 0);
            multiply(1, 0);
            write(n0 + kCols);
        }
    }
}

// dW, dH and db of a piece in one launch: small products end sooner than a launch begins
template <class K> struct PairParams {
    typedef typename K::E T;
    Params w, h;
    typename OutW<K>::Params ew;
    typename OutH<K>::Params eh;
    Bias<K> b;
    Few<K> few;
    unsigned blocks_w, blocks_h;
};
// SH: dH's tile.  ROWS: 0, or few rows' dW
template <class K, class SH, int ROWS> __global__ void __launch_bounds__(Small::kThreads, SH::kPerSimd) pair_kernel(const PairParams<K> p)
{
    static_assert(SH::kThreads == Small::kThreads, "one kernel");
    extern __shared__ __align__(1024) unsigned char smem[];
    typedef typename K::P P;
    unsigned block = blockIdx.x;
    if (block < p.blocks_h) { // (dH's sums are the longer ones: they begin first)
        mm_tile<P, Lay::kAlong, Lay::kDown, SH, OutH<K>>(p.h, p.eh, block, smem);
        return;
    }
    block -= p.blocks_h;
    if (block < p.blocks_w) {
        if constexpr (ROWS > 0) few_rows<K, ROWS>(p.few, block);
        else mm_tile<P, Lay::kDown, Lay::kDown, Small, OutW<K>>(p.w, p.ew, block, smem);
    } else {
        bias_sums(p.b, block - p.blocks_w, (float(*)[64])smem);
    }
}

// a slice's part of the logits' products, [slice][T][ld]
struct Logits : Ending {
    static constexpr bool kCountsM = true;
    struct Params { float *out; int T, ld; };
    template <int MI, int NI> static __device__ __forceinline__ void run(const Params &e, const f32x16 (&acc)[MI][NI], const Place &p)
    {
        typedef RowBlock<Fmt::kF32, NI> Block;
#pragma unroll
        for (int i = 0; i < MI; ++i) {
            const int m0 = p.m0 + i * 32;
            put_scaled(acc, i, Factor<false>(1.f, 0), p);
            Block::each(p.lds, p.lane, [&](int row, int at, u32x4 x) {
                if (m0 + row < p.M && p.n0 + at / 4 < e.ld) *(u32x4 *)(e.out + ((long)p.slice * e.T + m0 + row) * e.ld + p.n0 + at / 4) = x;
            });
        }
    }
};
// ... joined: four logits of row m
template <class K> __device__ __forceinline__ void join_logits(const float *part, long slice_stride, int slices, const typename K::E *b, int n, int V, int ze, float (&z)[4])
{
    float bias[4];
    load_bias(b, n, V, bias);
    f32x4 s = {0.f, 0.f, 0.f, 0.f};
    for (int k0 = 0; k0 < slices; k0 += 8) { // eight slices on their way at a time
        f32x4 x[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) x[k] = k0 + k < slices ? *(const f32x4 *)(part + (k0 + k) * slice_stride + n) : f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int k = 0; k < 8; ++k) s += x[k];
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) z[e] = n + e < V ? (K::kSplit ? ldexpf(s[e], ze) : s[e]) + bias[e] : -INFINITY;
}
// loss and lse of a compact row from the slices' logits, a block to a row
template <class K> __global__ void __launch_bounds__(256)
row_loss_kernel(const Meta meta, const float *__restrict__ part, long slice_stride, int ld, int slices, const typename K::E *__restrict__ b, int V,
                float *__restrict__ loss, float *__restrict__ lse)
{
    const int m = blockIdx.x;
    if (m >= meta.rows()) return;
    const int label = meta.label_of(m), t = meta.row_of(m);
    if (label == Meta::kOut) {
        if (threadIdx.x == 0) loss[t] = lse[t] = 0.f;
        return;
    }
    const int ze = K::kSplit ? -(meta.exps[0] + meta.exps[1]) : 0;
    const float *row = part + (long)m * ld;
    float top = -INFINITY, sum = 0.f;
    __shared__ float at_label, tops[4], sums[4];
    for (int n = threadIdx.x * 4; n < V; n += 1024) {
        float z[4];
        join_logits<K>(row, slice_stride, slices, b, n, V, ze, z);
        float m4 = fmaxf(fmaxf(z[0], z[1]), fmaxf(z[2], z[3]));
        if (label >= n && label < n + 4) at_label = label == n ? z[0] : label == n + 1 ? z[1] : label == n + 2 ? z[2] : z[3];
        m4 = fmaxf(m4, top);
        const float shift = m4 == -INFINITY ? 0.f : m4;
        sum *= __builtin_amdgcn_exp2f((top - shift) * kLog2e);
#pragma unroll
        for (int e = 0; e < 4; ++e) sum += __builtin_amdgcn_exp2f((z[e] - shift) * kLog2e);
        top = m4;
    }
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const float wtop = wave_max(top);
    sum *= __builtin_amdgcn_exp2f((top - (wtop == -INFINITY ? 0.f : wtop)) * kLog2e);
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) sum += __shfl_xor(sum, off, 64);
    if (lane == 0) {
        tops[wave] = wtop;
        sums[wave] = sum;
    }
    __syncthreads();
    if (threadIdx.x == 0) {
        top = fmaxf(fmaxf(tops[0], tops[1]), fmaxf(tops[2], tops[3]));
        const float shift = top == -INFINITY ? 0.f : top;
        sum = 0.f;
        for (int w = 0; w < 4; ++w) sum += sums[w] * __builtin_amdgcn_exp2f((tops[w] - shift) * kLog2e);
        const float l = top + logf(sum);
        lse[t] = l;
        loss[t] = at_label == -INFINITY ? INFINITY : l - at_label;
    }
}
// G, four neighbours to a thread: of two halves 16 rows by 64 classes to a block, which has a largest number for each, else 1024 of a row.  AGAIN: as Grad's
template <class K> constexpr int kGradRows = K::kSplit ? 16 : 1;
template <class K, bool AGAIN> __global__ void __launch_bounds__(256)
row_grad_kernel(const Meta meta, const float *__restrict__ part, long slice_stride, int ld, int slices, const typename K::E *__restrict__ b, int V,
                char *__restrict__ G, long ld_g, bool rests, uint32_t *__restrict__ peak)
{
    constexpr int kThreads = 256 / kGradRows<K>; // of a row
    const int lane = threadIdx.x & 63, m = blockIdx.x * kGradRows<K> + threadIdx.x / kThreads, n = (blockIdx.y * kThreads + threadIdx.x % kThreads) * 4;
    const float largest = meta.largest(lane);
    if (AGAIN && !formed_again(meta, peak, blockIdx.y * 64, min(V - (int)blockIdx.y * 64, 64), lane)) return;
    float g[4] = {0.f, 0.f, 0.f, 0.f};
    if (m < meta.rows() && n < ((V + 7) & ~7)) {
        const int label = meta.label_of(m);
        const float q = meta.q_of(m, largest), lse = meta.lse_of(m);
        if (label != Meta::kOut && n < V) {
            const int ze = K::kSplit ? -(meta.exps[0] + meta.exps[1]) : 0;
            float z[4];
            join_logits<K>(part + (long)m * ld, slice_stride, slices, b, n, V, ze, z);
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (n + e < V) g[e] = q * (__builtin_amdgcn_exp2f((z[e] - lse) * kLog2e) - (n + e == label ? 1.f : 0.f));
        }
        if (AGAIN) {
            const float v[4] = {ldexpf(g[0], -peak_exp(peak[min(n, V - 1)])), ldexpf(g[1], -peak_exp(peak[min(n + 1, V - 1)])),
                                ldexpf(g[2], -peak_exp(peak[min(n + 2, V - 1)])), ldexpf(g[3], -peak_exp(peak[min(n + 3, V - 1)]))};
            store_gradient<K>(G + (long)m * ld_g, n, v);
        } else if (K::kSplit) {
            const int e = -row_exp(q);
            const float v[4] = {ldexpf(g[0], e), ldexpf(g[1], e), ldexpf(g[2], e), ldexpf(g[3], e)};
            store_gradient<K>(G + (long)m * ld_g, n, v);
        } else {
            store_gradient<K>(G + (long)m * ld_g, n, g);
        }
        if (K::kG == Fmt::kBf16 && rests) {
            const float r[4] = {rest_of(g[0]), rest_of(g[1]), rest_of(g[2]), rest_of(g[3])};
            store_gradient<K>(G + (long)(m + kLoRow) * ld_g, n, r);
        }
    }
    if constexpr (K::kSplit && !AGAIN) { // the classes' largest of the block's rows
        __shared__ float tops[4][64];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            float v = fabsf(g[e]);
            v = fmaxf(v, __shfl_xor(v, 16, 64));
            v = fmaxf(v, __shfl_xor(v, 32, 64));
            if (lane < 16) tops[threadIdx.x >> 6][lane * 4 + e] = v;
        }
        __syncthreads();
        if (threadIdx.x < 64 && (int)(blockIdx.y * 64 + threadIdx.x) < V)
            raise_peak(peak + blockIdx.y * 64 + threadIdx.x, fmaxf(fmaxf(tops[0][lane], tops[1][lane]), fmaxf(tops[2][lane], tops[3][lane])));
    }
}

} // namespace

void plan_loss(const LossGeom &g, bool backward, LossPlan *p)
{
    // Few rows (and short forward passes): everything is read where it lies.  With more of them the float instruction costs more than the
    // passes that compact rows, find the largest numbers and split everything beforehand.  Packed beforehand and as they lie, both passes:
    //   bfloat16  16 x 256 x 300  28 and 23 us    64 x 700 x 5000  53 and 40 us    64 x 2048 x 30000  152 and 106 us
    //   float     40 x 256 x 300  39 and 34 us    64 x 2048 x 600  52 and 38 us    64 x 2048 x 30000  564 and 365 us
    //            128 x 1024 x 1000  52 and 40 us  128 x 700 x 5000  69 and 77 us   128 x 1001 x 20000  223 and 262 us
    // Forward passes of float read a large operand once so, where the other has few rows, and small ones save two launches: 128 x 2048 x
    // 30000  234 and 151 us, 12000 x 4000 x 64  193 and 88, 300 x 256 x 300  18 and 13, 1000 x 512 x 1000  25 and 19, 2000 x 1000 x 1000  44 and 47.
    // Short ones of bfloat16 save the launch that packs, though rows that are left out are multiplied then (512 x 1024 x 8000
    // 28 and 21 us, with half of them left out 26 and 21; 256 x 512 x 21841  28 and 25, 22 and 24).
    const double volume = (double)g.T * g.D * g.V;
    const int in4 = g.dtype == CAC_F32 ? 1 : 2; // numbers in 4 bytes
    if (backward) p->few = g.T <= kFewRows || (g.dtype == CAC_F32 && g.T <= kFewFloatRows && (double)g.D * g.V <= 2e6);
    else if (g.dtype == CAC_F32) p->few = g.T <= kFewFloatRows || g.V <= kFewFloatRows || volume <= 1e9;
    else p->few = g.T <= kFewRows || (volume <= 5e9 && g.D % 8 == 0 && g.ld_h % 8 == 0 && g.ld_w % 8 == 0);
    p->direct = p->few && g.D % in4 == 0 && g.ld_h % in4 == 0 && g.ld_w % in4 == 0;
    p->odd = p->direct && (g.D % (4 * in4) || g.ld_h % (4 * in4) || g.ld_w % (4 * in4));
    p->raw = g.dtype == CAC_F32 && p->few;
    p->rests = p->few && !p->raw && g.T <= kLoRow;
    p->split = g.dtype == CAC_F32 && !p->raw;
    p->pack_w = !p->direct && (p->split || g.D % 8 || g.ld_w % 8);
    p->dp = (g.D + 7) / 8 * 8;
    const int e = g.dtype == CAC_F32 ? 4 : 2; // bytes of a number, as it lies, in two halves, and of G
    p->row_bytes = e * p->dp;
    // A piece's G and packed weights take 1 GiB at most, the weights alone half of that, or 4096 classes; where one launch forms dW and dH of
    // float, G as it is formed again lies beside it (apart, which would spare that, 4000 x 64 x 20000 takes 523 us and not 463: db's sums
    // have nothing to run beside).  Smaller pieces cost more ends of launches and more sums of dH to add to: 4096 x 1024 x 32000 float
    // 3.49 ms in pieces of 256 MiB, 3.08 of 1 GiB, 3.06 in one; 2048 x 1024 x 200000 float forward 2.88 ms of 256 MiB, 2.75 of 512, 2.66 in one.
    const long per_class = (backward ? g.T * e : 0) + (p->pack_w ? p->row_bytes : 0);
    long piece = per_class ? ((backward ? 1024L : 512L) << 20) / per_class / 256 * 256 : g.V;
    if (piece < 4096) piece = 4096;
    if (piece > 1L << 19) piece = 1L << 19;
    if (piece >= g.V) piece = g.V;
    while (!fits_grid(kBig, tiles_of(kBig, g.T, piece, false))) piece /= 2; // (millions of rows)
    p->pieces = (int)((g.V + piece - 1) / piece);
    if (p->pieces > 1) piece = ((g.V + p->pieces - 1) / p->pieces + 255) / 256 * 256;
    p->pieces = (int)((g.V + piece - 1) / piece);
    p->piece = piece;
    // A sum over D in slices leaves its parts of the logits in the workspace (256 x 8192 x 2000 float forward: 107 us in one, 82 so).
    const long logits = g.T * ((piece + 3) & ~3L) * 4;
    const Format f = p->raw ? kRaw : p->split ? kSplit : kBf16;
    p->z = choose(f, g.T, piece, 1, g.D, false, p->pieces > 1 ? 1 : 16, p->raw || g.T <= kFewRows);
    p->w = choose(f, piece, g.D, 1, g.T, false, 1);
    p->h = choose(f, g.T, g.D, 1, piece, false, 128);
    // dW and dH together, in the smallest tiles, where both would take them anyway or there is little to multiply: one launch, and one
    // end where compute units run out of work (512 x 512 x 1500 float 68 us apart, 55 so; 1024 x 1024 x 8000 bfloat16 145 and 134,
    // 1024 x 2048 x 16000 341 and 379).
    const double work = 4.0 * g.T * g.D * piece * (p->split ? 3 : 1);
    p->pair = backward && (p->few || work < 7e10 || (p->w.shape == kSmall && p->h.shape == kSmall));
    if (p->pair) {
        p->w = Choice{kSmall, 1};
        p->h = choose(f, g.T, g.D, 1, piece, false, 128, true);
    }
    p->parts = 0;
    for (int k = 0; k < p->pieces; ++k) p->parts += wave_columns(k + 1 < p->pieces ? piece : g.V - (p->pieces - 1) * piece, p->z.shape);
    size_t o = 0;
    p->o_meta = o;
    o += meta_bytes(g.T);
    p->o_h = o;
    if (!p->direct) o += up256((size_t)g.T * p->row_bytes);
    p->o_w = o;
    if (p->pack_w) o += up256((size_t)piece * p->row_bytes);
    p->o_part = o;
    if (!backward && p->z.slices == 1) o += up256((size_t)p->parts * 2 * g.T * 4);
    p->o_z = o;
    if (p->z.slices > 1) o += up256((size_t)logits * p->z.slices);
    p->o_g = o;
    if (backward) o += up256((size_t)(g.T + (p->rests ? kLoRow : 0)) * ((piece + 7) / 8 * 8) * e);
    // (two halves: what classes with small G are formed again with; dW and dH of one launch read both)
    p->o_peak = o;
    if (backward && p->split) o += up256((size_t)piece * 4);
    p->o_again = p->o_g;
    if (p->split && p->pair) {
        p->o_again = o;
        o += up256((size_t)g.T * ((piece + 7) / 8 * 8) * e);
    }
    p->o_acc = o;
    if (backward && (p->pieces > 1 || p->h.slices > 1)) o += up256((size_t)p->h.slices * g.T * g.D * 4);
    p->bytes = o;
}

namespace {

template <class K> class Loss {
    typedef typename K::E T;
    typedef typename K::P P;
    static constexpr bool kDirect = P::kRaw || P::kUnit == 4; // always few rows
    const LossGeom &g;
    const LossPlan &p;
    const T *H, *W, *b;
    char *ws;
    hipStream_t st;
    Meta meta;
    int parts_h = 0, parts_w = 0;
    const void *h = nullptr, *w = nullptr; // the operands of the piece at hand
    long ld_h = 0, ld_w = 0;

    // How the products read H and the weights of classes v0 .. v0 + n; packs what has to be, H's rows with the first piece.
    hipError_t operands(long v0, long n, PackRows *rows)
    {
        const bool pack_h = v0 == 0 && !p.direct;
        h = p.direct ? (const void *)H : ws + p.o_h;
        ld_h = p.direct ? g.ld_h * (long)sizeof(T) : p.row_bytes;
        w = p.pack_w ? (const void *)(ws + p.o_w) : W + v0 * g.ld_w;
        ld_w = p.pack_w ? p.row_bytes : g.ld_w * (long)sizeof(T);
        if constexpr (kDirect) return hipSuccess; // (everything lies where it is)
        else return !pack_h && !p.pack_w ? hipSuccess : pack(v0, n, pack_h, rows);
    }
    hipError_t pack(long v0, long n, bool pack_h, PackRows *rows)
    {
        rows->H = H;
        rows->W = W + v0 * g.ld_w;
        rows->ld_h = g.ld_h;
        rows->ld_w = g.ld_w;
        rows->T = (int)g.T;
        rows->D = (int)g.D;
        rows->rows_per_block = (int)(g.T / 1024 < 4 ? 4 : g.T / 1024); // every block counts the labels before its own
        rows->row_blocks = pack_h ? cdiv(g.T, rows->rows_per_block) : 0;
        rows->classes = (int)n;
        rows->parts_h = parts_h;
        rows->parts_w = parts_w;
        rows->out = ws + p.o_h;
        rows->out_w = ws + p.o_w;
        rows->row_bytes = p.row_bytes;
        rows->meta = meta;
        const long waves = g.D <= kShortRow ? (n * ((g.D + 7) / 8) + 63) / 64 : n; // with something to do
        const long weight_blocks = !p.pack_w ? 0 : waves > 4 * 4096 ? 4096 : (waves + 3) / 4;
        hipLaunchKernelGGL(pack_kernel<K>, dim3((unsigned)(rows->row_blocks + weight_blocks)), dim3(256), 0, st, *rows);
        return hipGetLastError();
    }
    Params logits_params(long n) const
    {
        Params m{};
        m.a = h;
        m.lda = ld_h;
        m.b = w;
        m.ldb = ld_w;
        m.M = (int)g.T;
        m.N = (int)n;
        m.K = (int)g.D;
        m.batch = 1;
        if (p.few) m.counts_m = meta.counts;
        else m.m_dev = meta.count;
        return m;
    }
    long ld_logits() const { return (p.piece + 3) & ~3L; }
    hipError_t logits_in_slices(long n)
    {
        return launch<P, Lay::kAlong, Lay::kAlong, Logits>(logits_params(n), {(float *)(ws + p.o_z), (int)g.T, (int)ld_logits()}, p.z, st);
    }
    template <class SH, int ROWS> hipError_t launch_pair(PairParams<K> &q, bool want_h, int bias_blocks)
    {
        constexpr int lds = SH::kLds > Small::kLds ? SH::kLds : Small::kLds;
        if (!q.ew.out) {
            q.blocks_w = 0;
        } else if (ROWS) {
            const long blocks = cdiv(g.D, kFewColumns<K>), all = cdiv(q.few.V, 32) * blocks;
            const long run = all / 4096 < 1 ? 1 : all / 4096 > 16 ? 16 : all / 4096;
            q.few.run = (int)run;
            q.few.runs = cdiv(blocks, run);
            q.blocks_w = (unsigned)cdiv((long)cdiv(q.few.V, 32) * q.few.runs, 4);
        } else {
            q.blocks_w = place_tiles<Small>(&q.w, false, 1, kPass<P, Small::R>);
        }
        if (want_h) q.blocks_h = place_tiles<SH>(&q.h, false, p.h.slices, kPass<P, SH::R>);
        static const hipError_t attr =
            hipFuncSetAttribute(reinterpret_cast<const void *>(pair_kernel<K, SH, ROWS>), hipFuncAttributeMaxDynamicSharedMemorySize, lds);
        if (attr != hipSuccess) return attr;
        hipLaunchKernelGGL((pair_kernel<K, SH, ROWS>), dim3(q.blocks_w + q.blocks_h + bias_blocks), dim3(Small::kThreads), lds, st, q);
        return hipGetLastError();
    }
    template <class SH> hipError_t launch_few(PairParams<K> &q, bool want_h, int bias_blocks)
    {
        constexpr bool low = SH::TM == 32; // (float: the tile of up to 32 rows, and of no more)
        if constexpr (!P::kRaw || low) {
            if (g.T <= 16) return launch_pair<SH, 16>(q, want_h, bias_blocks);
            if (g.T <= 32) return launch_pair<SH, 32>(q, want_h, bias_blocks);
        }
        if constexpr (!low) {
            if (g.T <= 64) return launch_pair<SH, 64>(q, want_h, bias_blocks);
            if constexpr (P::kRaw) return launch_pair<SH, 128>(q, want_h, bias_blocks);
        }
        return hipErrorInvalidValue;
    }
    // G of classes v0 .. v0 + n; AGAIN: of those with small G
    template <bool AGAIN> hipError_t gradients(long v0, long n, char *G, long ld_g)
    {
        if constexpr (AGAIN && !K::kSplit) {
            return hipSuccess;
        } else {
            uint32_t *peak = p.split ? (uint32_t *)(ws + p.o_peak) : nullptr;
            if (p.z.slices == 1)
                return launch<P, Lay::kAlong, Lay::kAlong, Grad<K, AGAIN>>(logits_params(n), {b ? b + v0 : nullptr, meta, G, ld_g, (int)v0, p.rests, peak}, p.z, st);
            if (!AGAIN) { // (one piece; the logits stay where they are)
                const hipError_t e = logits_in_slices(n);
                if (e != hipSuccess) return e;
            }
            hipLaunchKernelGGL((row_grad_kernel<K, AGAIN>), dim3(cdiv(g.T, kGradRows<K>), cdiv(g.V, 1024 / kGradRows<K>)), dim3(256), 0, st, meta, (const float *)(ws + p.o_z),
                               g.T * ld_logits(), (int)ld_logits(), p.z.slices, b, (int)g.V, G, ld_g, p.rests, peak);
            return hipGetLastError();
        }
    }
    hipError_t launch_together(PairParams<K> &q, bool want_h, int bias_blocks)
    {
        if constexpr (K::kSplit) {
            return launch_pair<Small, 0>(q, want_h, bias_blocks);
        } else {
            if constexpr (!kDirect)
                if (!p.few) return launch_pair<Small, 0>(q, want_h, bias_blocks);
            if constexpr (P::kRaw)
                if (p.h.shape == kLow) return launch_few<Low>(q, want_h, bias_blocks);
            return launch_few<Small>(q, want_h, bias_blocks);
        }
    }
    hipError_t largest_magnitudes()
    {
        if (!p.split) return hipSuccess;
        parts_h = cdiv(g.T, 4) > kMaxParts ? kMaxParts : cdiv(g.T, 4);
        parts_w = cdiv(g.V, 4) > kMaxParts ? kMaxParts : cdiv(g.V, 4);
        hipLaunchKernelGGL(top_kernel, dim3(parts_h + parts_w), dim3(256), 0, st, (const float *)H, g.ld_h, g.T, (const float *)W, g.ld_w, g.V, g.D,
                           meta.counts, parts_h, meta.top, meta.uneven);
        return hipGetLastError();
    }

public:
    Loss(const LossGeom &g_, const LossPlan &p_, const void *H_, const void *W_, const void *b_, const int64_t *labels, void *ws_, hipStream_t st_)
        : g(g_), p(p_), H((const T *)H_), W((const T *)W_), b((const T *)b_), ws((char *)ws_), st(st_), meta(meta_at((char *)ws_ + p_.o_meta, g_.T))
    {
        meta.direct = p.few;
        meta.counts = Counts{labels, g.ignore, (int)g.V};
    }

    hipError_t forward(float *loss, float *lse)
    {
        hipError_t e = largest_magnitudes();
        if (e != hipSuccess) return e;
        PackRows rows{};
        rows.loss = loss;
        rows.lse_out = lse;
        float *part = (float *)(ws + p.o_part);
        int part0 = 0;
        for (long v0 = 0; v0 < g.V; v0 += p.piece) {
            const long n = v0 + p.piece < g.V ? p.piece : g.V - v0;
            if ((e = operands(v0, n, &rows)) != hipSuccess) return e;
            if (p.z.slices > 1) { // (one piece)
                if ((e = logits_in_slices(n)) != hipSuccess) return e;
                hipLaunchKernelGGL(row_loss_kernel<K>, dim3((unsigned)g.T), dim3(256), 0, st, meta, (const float *)(ws + p.o_z), g.T * ld_logits(),
                                   (int)ld_logits(), p.z.slices, b, (int)g.V, loss, lse);
                return hipGetLastError();
            }
            e = launch<P, Lay::kAlong, Lay::kAlong, Stats<K>>(logits_params(n), {b ? b + v0 : nullptr, meta, part, g.T, part0, (int)v0}, p.z, st);
            if (e != hipSuccess) return e;
            part0 += (int)wave_columns(n, p.z.shape);
        }
        // Few rows of many parts: a block to a row; else sixteen rows, whose parts lie side by side (forward, in blocks of one row and of
        // sixteen: 64 x 256 x 50000 20 and 25 us, 64 x 256 x 4000 9.9 and 9.3, 1024 x 256 x 50000 99 and 88).
        if (g.T <= 256 && p.parts > 128) hipLaunchKernelGGL(join_kernel<1>, dim3((unsigned)g.T), dim3(256), 0, st, meta, (const float *)part, (int)p.parts, g.T, loss, lse);
        else hipLaunchKernelGGL(join_kernel<16>, dim3(cdiv(g.T, 16)), dim3(256), 0, st, meta, (const float *)part, (int)p.parts, g.T, loss, lse);
        return hipGetLastError();
    }

    hipError_t backward(const float *lse, const float *gloss, T *dH, T *dW, T *db)
    {
        hipError_t e = largest_magnitudes();
        if (e != hipSuccess) return e;
        meta.lse_in = lse;
        meta.gloss = gloss;
        PackRows rows{};
        rows.lse = lse;
        rows.gloss = gloss;
        rows.dH = p.few ? nullptr : dH;
        rows.peak = p.split ? (uint32_t *)(ws + p.o_peak) : nullptr;
        char *const G = ws + p.o_g, *const again = ws + p.o_again;
        const uint32_t *const peak = rows.peak;
        const long ld_g = (p.piece + 7) / 8 * 8 * (long)sizeof(T);
        float *sums = p.pieces > 1 || p.h.slices > 1 ? (float *)(ws + p.o_acc) : nullptr;
        for (long v0 = 0; v0 < g.V; v0 += p.piece) {
            const long n = v0 + p.piece < g.V ? p.piece : g.V - v0;
            if ((e = operands(v0, n, &rows)) != hipSuccess) return e;
            if ((e = gradients<false>(v0, n, G, ld_g)) != hipSuccess) return e;
            PairParams<K> q{};
            q.w.a = G;
            q.w.lda = ld_g;
            q.w.b = h;
            q.w.ldb = ld_h;
            q.w.M = (int)n;
            q.w.N = (int)g.D;
            q.w.K = (int)g.T;
            q.w.batch = 1;
            q.w.k_dev = meta.count;
            q.ew = {dW ? dW + v0 * g.D : nullptr, meta, peak, again == G ? nullptr : again};
            q.h.a = G;
            q.h.lda = ld_g;
            q.h.b = w;
            q.h.ldb = ld_w;
            q.h.M = (int)g.T + (p.rests ? kLoRow : 0);
            q.h.N = (int)g.D;
            q.h.K = (int)n;
            q.h.batch = 1;
            if (!p.few) q.h.m_dev = meta.count;
            q.eh = {dH, sums, g.T * g.D, v0 > 0, p.rests, meta};
            q.b = {meta, G, ld_g, (int)n, db ? db + v0 : nullptr, p.rests, peak, q.ew.again};
            const int bias_blocks = db ? cdiv(n, 64) : 0;
            if (p.pair) {
                if (K::kSplit && (dW || db) && (e = gradients<true>(v0, n, again, ld_g)) != hipSuccess) return e;
                q.few = {meta, G, (const T *)h, ld_g, ld_h, (int)n, (int)g.D, q.ew.out, 0, 0};
                // dH may take the place of H; where H is read as it lies dW has to be done with it by then
                if (p.direct && (const T *)dH == H && (dW || db)) {
                    e = launch_together(q, false, bias_blocks);
                    q.ew.out = nullptr;
                    if (e == hipSuccess) e = launch_together(q, true, 0);
                } else {
                    e = launch_together(q, dH, bias_blocks);
                }
            } else if constexpr (!kDirect) {
                // (G of two halves as it is formed first is what dH takes, as it is formed again what dW does)
                if (dH) e = launch<P, Lay::kAlong, Lay::kDown, OutH<K>>(q.h, q.eh, p.h, st);
                if (K::kSplit && (dW || db) && e == hipSuccess) e = gradients<true>(v0, n, G, ld_g);
                if (dW && e == hipSuccess) e = launch<P, Lay::kDown, Lay::kDown, OutW<K>>(q.w, q.ew, p.w, st);
                if (db && e == hipSuccess) {
                    hipLaunchKernelGGL(bias_kernel<K>, dim3(bias_blocks), dim3(256), 0, st, q.b);
                    e = hipGetLastError();
                }
            }
            if (e != hipSuccess) return e;
        }
        if (dH && sums) {
            // (1 x 512 x 21841: 51 us where every thread adds up all of its slices, 46 where waves share them; one slice of 8192 x 4096:
            // 7.95 and 8.05 ms of the whole)
            if (p.h.slices >= 8)
                hipLaunchKernelGGL((finish_rows_kernel<T, true>), dim3((unsigned)g.T, cdiv(g.D, 256)), dim3(256), 0, st, meta, (const float *)sums,
                                   g.T * g.D, p.h.slices, (int)g.D, dH);
            else
                hipLaunchKernelGGL((finish_rows_kernel<T, false>), dim3((unsigned)g.T, cdiv(g.D, 1024)), dim3(256), 0, st, meta, (const float *)sums,
                                   g.T * g.D, p.h.slices, (int)g.D, dH);
            e = hipGetLastError();
        }
        return e;
    }
};

} // namespace

hipError_t launch_loss_fwd(const LossGeom &g, const LossPlan &p, const void *H, const void *W, const void *b, const int64_t *labels,
                           float *loss, float *lse, void *ws, hipStream_t st)
{
    if (p.raw && p.odd) return Loss<OfRaw<RawOdd>>(g, p, H, W, b, labels, ws, st).forward(loss, lse);
    if (p.raw) return Loss<OfRaw<Raw>>(g, p, H, W, b, labels, ws, st).forward(loss, lse);
    if (p.split) return Loss<OfSplit>(g, p, H, W, b, labels, ws, st).forward(loss, lse);
    if (p.odd) return Loss<OfBf16<Bf16Odd>>(g, p, H, W, b, labels, ws, st).forward(loss, lse);
    return Loss<OfBf16<Bf16>>(g, p, H, W, b, labels, ws, st).forward(loss, lse);
}

hipError_t launch_loss_bwd(const LossGeom &g, const LossPlan &p, const void *H, const void *W, const void *b, const int64_t *labels,
                           const float *lse, const float *gloss, void *dH, void *dW, void *db, void *ws, hipStream_t st)
{
    if (p.raw && p.odd) return Loss<OfRaw<RawOdd>>(g, p, H, W, b, labels, ws, st).backward(lse, gloss, (float *)dH, (float *)dW, (float *)db);
    if (p.raw) return Loss<OfRaw<Raw>>(g, p, H, W, b, labels, ws, st).backward(lse, gloss, (float *)dH, (float *)dW, (float *)db);
    if (p.split) return Loss<OfSplit>(g, p, H, W, b, labels, ws, st).backward(lse, gloss, (float *)dH, (float *)dW, (float *)db);
    if (p.odd) return Loss<OfBf16<Bf16Odd>>(g, p, H, W, b, labels, ws, st).backward(lse, gloss, (bf16_t *)dH, (bf16_t *)dW, (bf16_t *)db);
    return Loss<OfBf16<Bf16>>(g, p, H, W, b, labels, ws, st).backward(lse, gloss, (bf16_t *)dH, (bf16_t *)dW, (bf16_t *)db);
}

} // namespace cac
