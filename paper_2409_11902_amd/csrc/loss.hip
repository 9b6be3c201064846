// Softmax cross entropy of a linear classifier, z = H W^T + b, over many classes.  Neither pass keeps the logits:
//
//   forward : lse_t = log sum_v exp z_tv from each tile's maximum and sum of a row, loss_t = lse_t - z_t,label
//   backward: the logits once more, piece of the classes by piece, G_tv = q_t (exp(z_tv - lse_t) - [v = label_t]) from them, then
//             dW = c G^T H and dH = c G W; the rows' gradients are c q_t, c the largest of them, so that a mean's are q = 1 exactly
//             and G is rounded once.
//
// Rows that are left out (label equal to ignore_index, or no class) are taken out of H when it is copied into the workspace: no
// product reads them, whatever stands there, and the products get shorter by them.
// Sums are of 32 bits; G is rounded to bfloat16 for bfloat16 operands (its products' operands are), and held as two halves for float.
#include "mm_core.h"
#include "train_ends.h"

namespace cac {

namespace {

using namespace mm;

constexpr float kLog2e = 1.44269504088896340736f;
constexpr int kStoreG = 14;        // G is stored times 2^14 as two halves: |G| <= 1, and 1e-8 is still a normal number
constexpr int kMaxParts = 512;     // blocks that look for a matrix's largest number

// What the passes over compact rows know about them.
struct Meta {
    int *count;       // [0]: rows that count
    int *exps;        // H and W are stored times 2^exps[0] and 2^exps[1] as two halves
    float *c;         // [0]: the largest of the rows' gradients
    int *row;         // compact row -> row of H
    int *label;
    float *q, *lse;
    float *zlabel;    // forward: the label's logit
    float *top;       // kMaxParts of H, then of W: largest magnitudes
};
__host__ __device__ inline size_t up256(size_t n) { return (n + 255) & ~(size_t)255; }
__host__ __device__ inline size_t meta_bytes(long T) { return 256 + up256(2 * kMaxParts * 4) + 5 * up256(4 * (size_t)T); }
inline Meta meta_at(char *p, long T)
{
    Meta m;
    const size_t n = up256(4 * (size_t)T);
    m.count = (int *)p;
    m.exps = (int *)(p + 64);
    m.c = (float *)(p + 128);
    m.top = (float *)(p + 256);
    p += 256 + up256(2 * kMaxParts * 4);
    m.row = (int *)p;
    m.label = (int *)(p + n);
    m.q = (float *)(p + 2 * n);
    m.lse = (float *)(p + 3 * n);
    m.zlabel = (float *)(p + 4 * n);
    return m;
}

__device__ __forceinline__ bool counts(int64_t label, int64_t ignore, long V) { return label != ignore && label >= 0 && label < V; }

__device__ __forceinline__ float wave_max(float v)
{
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) v = fmaxf(v, __shfl_xor(v, off, 64));
    return v;
}
__device__ __forceinline__ int wave_add(int v)
{
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) v += __shfl_xor(v, off, 64);
    return v;
}

// Largest finite magnitude of H (rows that count) and of W, a part from every block.
__global__ void __launch_bounds__(256) top_kernel(const float *__restrict__ H, long ld_h, long T, const float *__restrict__ W, long ld_w, long V,
                                                  long D, const int64_t *__restrict__ labels, int64_t ignore, int blocks_h, float *__restrict__ top)
{
    const bool is_h = (int)blockIdx.x < blocks_h;
    const int block = is_h ? blockIdx.x : blockIdx.x - blocks_h, blocks = is_h ? blocks_h : gridDim.x - blocks_h;
    const float *x = is_h ? H : W;
    const long rows = is_h ? T : V, ld = is_h ? ld_h : ld_w;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    float m = 0.f;
    for (long r = (long)block * 4 + wave; r < rows; r += blocks * 4) {
        if (is_h && !counts(labels[r], ignore, V)) continue;
        const float *p = x + r * ld;
        long d = lane;
        for (; d + 192 < D; d += 256) {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const float v = fabsf(p[d + e * 64]);
                m = v <= 3.4028235e38f ? fmaxf(m, v) : m;
            }
        }
        for (; d < D; d += 64) {
            const float v = fabsf(p[d]);
            m = v <= 3.4028235e38f ? fmaxf(m, v) : m;
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
    float m = 0.f;
    for (int i = threadIdx.x & 63; i < parts; i += 64) m = fmaxf(m, top[i]);
    m = wave_max(m);
    if (!(m > 0.f)) return 0;
    int e;
    frexpf(m, &e); // m < 2^e
    return min(14 - e, 120);
}

struct PackRows {
    const void *H;
    const int64_t *labels;
    int64_t ignore;
    long ld_h;
    int T, D, V;
    int rows_per_block;
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

// eight neighbours of a row of memory in float, zeros past its end
template <typename T> __device__ __forceinline__ void load8(const T *p, int n, int D, bool aligned, float (&v)[8])
{
    if (aligned && n + 8 <= D) {
        struct alignas(16) Some { T v[16 / sizeof(T)]; };
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
}
// ... and into a packed row (bfloat16: as they are; float: two halves, times `scale`)
__device__ __forceinline__ void store8(bf16_t, char *row, int n, const float (&v)[8], float)
{
    u32x4 u;
#pragma unroll
    for (int e = 0; e < 4; ++e) u[e] = f32x2_to_bf16x2(v[2 * e], v[2 * e + 1]);
    *(u32x4 *)(row + n * 2) = u;
}
__device__ __forceinline__ void store8(float, char *row, int n, const float (&v)[8], float scale)
{
#pragma unroll
    for (int h = 0; h < 8; h += 4) {
        const float x[4] = {v[h] * scale, v[h + 1] * scale, v[h + 2] * scale, v[h + 3] * scale};
        store_split(row, n + h, x);
    }
}

// Rows that count, one behind the other, and what is known about them.  A block takes a run of rows; where they go follows from the
// labels before them.
template <typename T> __global__ void __launch_bounds__(256) pack_rows_kernel(const PackRows p)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int first = blockIdx.x * p.rows_per_block, last = min(p.T, first + p.rows_per_block);
    __shared__ int red_n[4];
    __shared__ float red_c[4];
    int before = 0;
    float c = 0.f;
    for (int t = threadIdx.x; t < (p.gloss ? p.T : first); t += 256) {
        const bool in = counts(p.labels[t], p.ignore, p.V);
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
    const int exp_h = sizeof(T) == 4 ? stored_exp(p.meta.top, p.parts_h) : 0;
    const float scale = ldexpf(1.f, exp_h);
    if (blockIdx.x == 0 && wave == 0) {
        const int exp_w = sizeof(T) == 4 ? stored_exp(p.meta.top + kMaxParts, p.parts_w) : 0;
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
        const int64_t label = t < last ? p.labels[t] : 0;
        const bool in = t < last && counts(label, p.ignore, p.V);
        const uint64_t mask = __ballot(in);
        const int j = place + __popcll(mask & (((uint64_t)1 << lane) - 1));
        if (wave == 0 && t < last) {
            if (in) {
                p.meta.row[j] = t;
                p.meta.label[j] = (int)label;
                if (p.gloss) {
                    const float l = p.lse[t];
                    p.meta.q[j] = c > 0.f ? p.gloss[t] / c : p.gloss[t];
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
                const int jj = place + __popcll(mask & (((uint64_t)1 << k) - 1));
                const T *h = (const T *)p.H + (long)row * p.ld_h;
                char *o = p.out + (long)jj * p.row_bytes;
                for (int n = lane * 8; n < p.D; n += 512) {
                    float v[8];
                    load8(h, n, p.D, aligned, v);
                    store8(T(), o, n, v, scale);
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
template <typename T> __global__ void __launch_bounds__(256)
pack_weights_kernel(const T *__restrict__ W, long ld, int rows, int D, const int *__restrict__ exps, char *__restrict__ out, long row_bytes)
{
    const float s = sizeof(T) == 4 ? ldexpf(1.f, exps[1]) : 1.f;
    const int per_row = (D + 7) / 8;
    const bool aligned = ((uintptr_t)W & 15) == 0 && (ld * sizeof(T)) % 16 == 0;
    for (long c = (long)blockIdx.x * 256 + threadIdx.x; c < (long)rows * per_row; c += (long)gridDim.x * 256) {
        const int row = (int)(c / per_row), n = (int)(c - (long)row * per_row) * 8;
        float v[8];
        load8(W + row * ld, n, D, aligned, v);
        store8(T(), out + row * row_bytes, n, v, s);
    }
}

// four neighbours of b from n on, zeros past its end
template <typename T> __device__ __forceinline__ void load_bias(const T *b, int n, int N, float (&v)[4])
{
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = b && n + e < N ? Elem<T>::load(b + n + e) : 0.f;
}

// ---- endings of the products
// forward: maximum and sum of exp of a row over a wave's columns, and the label's logit
template <typename T> struct Stats {
    static constexpr bool kSymmetric = false;
    struct Params {
        const T *b;
        Meta meta;
        float *part;      // [2 * parts][T]
        long T_rows;
        int part0, v0;    // the piece's first part, its first class
    };
    template <int MI, int NI> static __device__ __forceinline__ void run(const Params &e, const f32x16 (&acc)[MI][NI], const Place &p)
    {
        const int ze = sizeof(T) == 4 ? -(e.meta.exps[0] + e.meta.exps[1]) : 0;
        const int part = e.part0 + p.part;
#pragma unroll
        for (int i = 0; i < MI; ++i) {
            const int m = p.m0 + i * 32 + (p.lane & 31);
            const int label = m < p.M ? e.meta.label[m] - e.v0 : -1;
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
                        const float v = (sizeof(T) == 4 ? ldexpf(acc[i][j][q * 4 + k], ze) : acc[i][j][q * 4 + k]) + bias[k];
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

// lse and loss of a compact row from its parts: 16 rows to a block, 16 threads to a row
__global__ void __launch_bounds__(256) join_kernel(const Meta meta, const float *__restrict__ part, int parts, long T_rows, float *__restrict__ loss,
                                                   float *__restrict__ lse)
{
    const int count = *meta.count;
    const int r = threadIdx.x & 15, s = threadIdx.x >> 4;
    const int j = blockIdx.x * 16 + r;
    float top = -INFINITY, sum = 0.f;
    if (j < count)
        for (int k0 = s; k0 < parts; k0 += 128) { // eight parts on their way at a time
            float t[8], u[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const int k = k0 + e * 16;
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
    __shared__ float tops[16][17], sums[16][17];
    tops[s][r] = top;
    sums[s][r] = sum;
    __syncthreads();
    if (s == 0 && j < count) {
        for (int k = 1; k < 16; ++k) top = fmaxf(top, tops[k][r]);
        const float shift = top == -INFINITY ? 0.f : top;
        float total = 0.f;
        for (int k = 0; k < 16; ++k) total += sums[k][r] * __builtin_amdgcn_exp2f((tops[k][r] - shift) * kLog2e);
        const float l = top + logf(total), z = meta.zlabel[j];
        const int t = meta.row[j];
        lse[t] = l;
        loss[t] = z == -INFINITY ? INFINITY : l - z; // (a masked label's loss, also where every class is masked)
    }
}

// backward: G of a piece
template <typename T> struct Grad {
    static constexpr bool kSymmetric = false;
    struct Params {
        const T *b;
        Meta meta;
        char *out;
        long ld;
        int v0;
    };
    template <int MI, int NI> static __device__ __forceinline__ void run(const Params &e, const f32x16 (&acc)[MI][NI], const Place &p)
    {
        const int ze = sizeof(T) == 4 ? -(e.meta.exps[0] + e.meta.exps[1]) : 0;
        const int Np = (p.N + 7) & ~7;
#pragma unroll
        for (int i = 0; i < MI; ++i) {
            const int m = p.m0 + i * 32 + (p.lane & 31);
            if (m >= p.M) continue;
            const int label = e.meta.label[m] - e.v0;
            const float q_row = e.meta.q[m], lse = e.meta.lse[m];
            char *row = e.out + (long)m * e.ld;
#pragma unroll
            for (int j = 0; j < NI; ++j)
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const int n = p.n0 + j * 32 + q * 8 + (p.lane >> 5) * 4;
                    if (n >= Np) continue;
                    float bias[4], g[4];
                    load_bias(e.b, n, p.N, bias);
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        const float z = (sizeof(T) == 4 ? ldexpf(acc[i][j][q * 4 + k], ze) : acc[i][j][q * 4 + k]) + bias[k];
                        const float x = q_row * (__builtin_amdgcn_exp2f((z - lse) * kLog2e) - (n + k == label ? 1.f : 0.f));
                        g[k] = n + k < p.N ? x : 0.f;
                    }
                    if (sizeof(T) == 4) {
#pragma unroll
                        for (int k = 0; k < 4; ++k) g[k] *= (float)(1 << kStoreG);
                        store_split(row, n, g);
                    } else {
                        u32x2 u;
                        u[0] = f32x2_to_bf16x2(g[0], g[1]);
                        u[1] = f32x2_to_bf16x2(g[2], g[3]);
                        *(u32x2 *)(row + n * 2) = u;
                    }
                }
        }
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

// dW of a piece
template <typename T> struct OutW {
    static constexpr bool kSymmetric = false;
    struct Params { T *out; Meta meta; };
    template <int MI, int NI> static __device__ __forceinline__ void run(const Params &e, const f32x16 (&acc)[MI][NI], const Place &p)
    {
        const float s = sizeof(T) == 4 ? ldexpf(*e.meta.c, -kStoreG - e.meta.exps[0]) : *e.meta.c;
        const bool wide = (p.N & 3) == 0;
#pragma unroll
        for (int i = 0; i < MI; ++i)
#pragma unroll
            for (int j = 0; j < NI; ++j)
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const int m = p.m0 + i * 32 + (p.lane & 31), n = p.n0 + j * 32 + q * 8 + (p.lane >> 5) * 4;
                    if (m >= p.M || n >= p.N) continue;
                    float v[4];
#pragma unroll
                    for (int k = 0; k < 4; ++k) v[k] = s * acc[i][j][q * 4 + k];
                    store_four(e.out + (long)m * p.N + n, n, p.N, wide, v);
                }
    }
};

// dH: the result, or sums of a slice (added to what the pieces before left)
template <typename T> struct OutH {
    static constexpr bool kSymmetric = false;
    struct Params { T *out; float *sums; long slice_stride; int add; Meta meta; };
    template <int MI, int NI> static __device__ __forceinline__ void run(const Params &e, const f32x16 (&acc)[MI][NI], const Place &p)
    {
        const float s = sizeof(T) == 4 ? ldexpf(*e.meta.c, -kStoreG - e.meta.exps[1]) : *e.meta.c;
        const bool wide = (p.N & 3) == 0;
#pragma unroll
        for (int i = 0; i < MI; ++i) {
            const int m = p.m0 + i * 32 + (p.lane & 31);
            if (m >= p.M) continue;
            const int row = e.sums ? m : e.meta.row[m];
#pragma unroll
            for (int j = 0; j < NI; ++j)
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const int n = p.n0 + j * 32 + q * 8 + (p.lane >> 5) * 4;
                    if (n >= p.N) continue;
                    float v[4];
#pragma unroll
                    for (int k = 0; k < 4; ++k) v[k] = s * acc[i][j][q * 4 + k];
                    if (!e.sums) {
                        store_four(e.out + (long)row * p.N + n, n, p.N, wide, v);
                        continue;
                    }
                    float *o = e.sums + p.slice * e.slice_stride + (long)m * p.N + n;
                    if (e.add)
#pragma unroll
                        for (int k = 0; k < 4; ++k)
                            if (n + k < p.N) v[k] += o[k];
                    store_four(o, n, p.N, wide, v);
                }
        }
    }
};

// dH from the slices' sums; a block takes 1024 numbers of a compact row
template <typename T> __global__ void __launch_bounds__(256)
finish_rows_kernel(const Meta meta, const float *__restrict__ sums, long slice_stride, int slices, int D, T *__restrict__ dH)
{
    if ((int)blockIdx.x >= *meta.count) return;
    const int n = blockIdx.y * 1024 + threadIdx.x * 4;
    if (n >= D) return;
    const long at = (long)blockIdx.x * D + n;
    const bool wide = (D & 3) == 0;
    float v[4] = {0.f, 0.f, 0.f, 0.f};
    for (int s = 0; s < slices; ++s) {
        const float *p = sums + s * slice_stride + at;
        if (wide) {
            const f32x4 x = *(const f32x4 *)p;
#pragma unroll
            for (int k = 0; k < 4; ++k) v[k] += x[k];
        } else {
#pragma unroll
            for (int k = 0; k < 4; ++k)
                if (n + k < D) v[k] += p[k];
        }
    }
    store_four(dH + (long)meta.row[blockIdx.x] * D + n, n, D, wide, v);
}

// db of a piece: the columns' sums of G, eight columns to a thread, the block's four waves over the rows
template <typename T> __global__ void __launch_bounds__(256)
bias_kernel(const Meta meta, const char *__restrict__ G, long ld, int V, T *__restrict__ db)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int count = *meta.count;
    // 8 chunks of columns by 8 rows to a wave
    const int chunk = blockIdx.x * 8 + (lane & 7), n = chunk * 8;
    float s[8] = {};
    if (n < V)
        for (int m = wave * 8 + (lane >> 3); m < count; m += 32) {
            const char *p = G + (long)m * ld + (long)chunk * (sizeof(T) == 4 ? 32 : 16);
            if (sizeof(T) == 4) {
                const f16x8 hi = *(const f16x8 *)p, lo = *(const f16x8 *)(p + 16);
#pragma unroll
                for (int e = 0; e < 8; ++e) s[e] += (float)hi[e] + (float)lo[e];
            } else {
                struct alignas(16) Eight { bf16_t v[8]; };
                const Eight v = *(const Eight *)p;
#pragma unroll
                for (int e = 0; e < 8; ++e) s[e] += bf16_to_f32(v.v[e]);
            }
        }
    __shared__ float red[4][64];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        s[e] += __shfl_xor(s[e], 8, 64);
        s[e] += __shfl_xor(s[e], 16, 64);
        s[e] += __shfl_xor(s[e], 32, 64);
        if (lane < 8) red[wave][lane * 8 + e] = s[e];
    }
    __syncthreads();
    if (threadIdx.x < 64 && (int)(blockIdx.x * 64 + threadIdx.x) < V) {
        const float c = sizeof(T) == 4 ? ldexpf(*meta.c, -kStoreG) : *meta.c;
        Elem<T>::store(db + blockIdx.x * 64 + threadIdx.x, c * (((red[0][lane] + red[1][lane]) + red[2][lane]) + red[3][lane]));
    }
}

} // namespace

void plan_loss(const LossGeom &g, bool backward, LossPlan *p)
{
    p->split = g.dtype == CAC_F32;
    p->dp = (g.D + 7) / 8 * 8;
    p->row_bytes = (p->split ? 4 : 2) * p->dp;
    p->pack_w = p->split || g.D % 8 || g.ld_w % 8;
    // A piece's G (and its packed weights) stay within half of the 256 MiB that the chip caches; at least 4096 classes, in whole tiles.
    const long per_class = (backward ? g.T * (p->split ? 4 : 2) : 0) + (p->pack_w ? p->row_bytes : 0);
    long piece = per_class ? (256L << 20) / per_class / 256 * 256 : g.V;
    if (piece < 4096) piece = 4096;
    if (piece > 1L << 19) piece = 1L << 19;
    if (piece >= g.V) piece = g.V;
    p->pieces = (int)((g.V + piece - 1) / piece);
    if (p->pieces > 1) piece = ((g.V + p->pieces - 1) / p->pieces + 255) / 256 * 256;
    p->pieces = (int)((g.V + piece - 1) / piece);
    p->piece = piece;
    p->z = choose(p->split, g.T, piece, 1, g.D, false, 1);
    p->w = choose(p->split, piece, g.D, 1, g.T, false, 1);
    p->h = choose(p->split, g.T, g.D, 1, piece, false, 16);
    p->parts = 0;
    for (int k = 0; k < p->pieces; ++k) p->parts += wave_columns(k + 1 < p->pieces ? piece : g.V - (p->pieces - 1) * piece, p->z.shape);
    size_t o = 0;
    p->o_meta = o;
    o += meta_bytes(g.T);
    p->o_h = o;
    o += up256((size_t)g.T * p->row_bytes);
    p->o_w = o;
    if (p->pack_w) o += up256((size_t)piece * p->row_bytes);
    p->o_part = o;
    if (!backward) o += up256((size_t)p->parts * 2 * g.T * 4);
    p->o_g = o;
    if (backward) o += up256((size_t)g.T * ((piece + 7) / 8 * 8) * (p->split ? 4 : 2));
    p->o_acc = o;
    if (backward && (p->pieces > 1 || p->h.slices > 1)) o += up256((size_t)p->h.slices * g.T * g.D * 4);
    p->bytes = o;
}

namespace {

// H's rows that count into the workspace, and what is known about them
template <typename T>
hipError_t launch_rows(const LossGeom &g, const LossPlan &p, const T *H, const T *W, const int64_t *labels, float *loss, float *lse_out,
                       const float *lse, const float *gloss, void *dH, char *ws, const Meta &meta, hipStream_t st)
{
    int parts_h = 0, parts_w = 0;
    if (p.split) {
        parts_h = (int)(g.T / 8 < 1 ? 1 : g.T / 8 > kMaxParts ? kMaxParts : g.T / 8);
        parts_w = (int)(g.V / 8 < 1 ? 1 : g.V / 8 > kMaxParts ? kMaxParts : g.V / 8);
        hipLaunchKernelGGL(top_kernel, dim3(parts_h + parts_w), dim3(256), 0, st, (const float *)H, g.ld_h, g.T, (const float *)W, g.ld_w, g.V, g.D,
                           labels, (int64_t)g.ignore, parts_h, meta.top);
    }
    PackRows r{};
    r.H = H;
    r.labels = labels;
    r.ignore = g.ignore;
    r.ld_h = g.ld_h;
    r.T = (int)g.T;
    r.D = (int)g.D;
    r.V = (int)g.V;
    r.rows_per_block = (int)(g.T / 1024 < 8 ? 8 : g.T / 1024); // every block counts the labels before its own
    r.parts_h = parts_h;
    r.parts_w = parts_w;
    r.out = ws + p.o_h;
    r.row_bytes = p.row_bytes;
    r.meta = meta;
    r.loss = loss;
    r.lse_out = lse_out;
    r.lse = lse;
    r.gloss = gloss;
    r.dH = dH;
    hipLaunchKernelGGL(pack_rows_kernel<T>, dim3(cdiv(g.T, r.rows_per_block)), dim3(256), 0, st, r);
    return hipGetLastError();
}

// classes v0 .. v0 + n of the weights as the products read them
template <typename T>
hipError_t piece_of_weights(const LossGeom &g, const LossPlan &p, const T *W, long v0, long n, const Meta &meta, char *ws, hipStream_t st,
                            const void **at, long *ld)
{
    const T *w = W + v0 * g.ld_w;
    if (!p.pack_w) {
        *at = w;
        *ld = g.ld_w * (long)sizeof(T);
        return hipSuccess;
    }
    const long chunks = n * ((g.D + 7) / 8);
    hipLaunchKernelGGL(pack_weights_kernel<T>, dim3((unsigned)(chunks > 256 * 4096 ? 4096 : (chunks + 255) / 256)), dim3(256), 0, st, w, g.ld_w, (int)n,
                       (int)g.D, (const int *)meta.exps, ws + p.o_w, p.row_bytes);
    *at = ws + p.o_w;
    *ld = p.row_bytes;
    return hipGetLastError();
}

template <typename T> struct FormatOf { typedef Bf16 type; };
template <> struct FormatOf<float> { typedef Split type; };

template <typename T>
hipError_t forward(const LossGeom &g, const LossPlan &p, const T *H, const T *W, const T *b, const int64_t *labels, float *loss, float *lse,
                   char *ws, hipStream_t st)
{
    typedef typename FormatOf<T>::type P;
    const Meta meta = meta_at(ws + p.o_meta, g.T);
    hipError_t e = launch_rows(g, p, H, W, labels, loss, lse, (const float *)nullptr, (const float *)nullptr, nullptr, ws, meta, st);
    if (e != hipSuccess) return e;
    float *part = (float *)(ws + p.o_part);
    int part0 = 0;
    for (long v0 = 0; v0 < g.V; v0 += p.piece) {
        const long n = v0 + p.piece < g.V ? p.piece : g.V - v0;
        Params m{};
        if ((e = piece_of_weights(g, p, W, v0, n, meta, ws, st, &m.b, &m.ldb)) != hipSuccess) return e;
        m.a = ws + p.o_h;
        m.lda = p.row_bytes;
        m.M = (int)g.T;
        m.N = (int)n;
        m.K = (int)g.D;
        m.m_dev = meta.count;
        m.batch = 1;
        e = launch<P, Lay::kAlong, Lay::kAlong, Stats<T>>(m, {b ? b + v0 : nullptr, meta, part, g.T, part0, (int)v0}, p.z, st);
        if (e != hipSuccess) return e;
        part0 += (int)wave_columns(n, p.z.shape);
    }
    hipLaunchKernelGGL(join_kernel, dim3(cdiv(g.T, 16)), dim3(256), 0, st, meta, (const float *)part, (int)p.parts, g.T, loss, lse);
    return hipGetLastError();
}

template <typename T>
hipError_t backward(const LossGeom &g, const LossPlan &p, const T *H, const T *W, const T *b, const int64_t *labels, const float *lse,
                    const float *gloss, T *dH, T *dW, T *db, char *ws, hipStream_t st)
{
    typedef typename FormatOf<T>::type P;
    const Meta meta = meta_at(ws + p.o_meta, g.T);
    hipError_t e = launch_rows(g, p, H, W, labels, nullptr, nullptr, lse, gloss, dH, ws, meta, st);
    if (e != hipSuccess) return e;
    char *G = ws + p.o_g;
    const long ld_g = (p.piece + 7) / 8 * 8 * (p.split ? 4 : 2);
    const bool sums = p.pieces > 1 || p.h.slices > 1;
    for (long v0 = 0; v0 < g.V; v0 += p.piece) {
        const long n = v0 + p.piece < g.V ? p.piece : g.V - v0;
        const void *w;
        long ld_w;
        if ((e = piece_of_weights(g, p, W, v0, n, meta, ws, st, &w, &ld_w)) != hipSuccess) return e;
        Params m{};
        m.a = ws + p.o_h;
        m.lda = p.row_bytes;
        m.b = w;
        m.ldb = ld_w;
        m.M = (int)g.T;
        m.N = (int)n;
        m.K = (int)g.D;
        m.m_dev = meta.count;
        m.batch = 1;
        e = launch<P, Lay::kAlong, Lay::kAlong, Grad<T>>(m, {b ? b + v0 : nullptr, meta, G, ld_g, (int)v0}, p.z, st);
        if (e != hipSuccess) return e;
        if (dW) {
            Params d{};
            d.a = G;
            d.lda = ld_g;
            d.b = ws + p.o_h;
            d.ldb = p.row_bytes;
            d.M = (int)n;
            d.N = (int)g.D;
            d.K = (int)g.T;
            d.k_dev = meta.count;
            d.batch = 1;
            e = launch<P, Lay::kDown, Lay::kDown, OutW<T>>(d, {dW + v0 * g.D, meta}, p.w, st);
            if (e != hipSuccess) return e;
        }
        if (dH) {
            Params d{};
            d.a = G;
            d.lda = ld_g;
            d.b = w;
            d.ldb = ld_w;
            d.M = (int)g.T;
            d.N = (int)g.D;
            d.K = (int)n;
            d.m_dev = meta.count;
            d.batch = 1;
            e = launch<P, Lay::kAlong, Lay::kDown, OutH<T>>(d, {dH, sums ? (float *)(ws + p.o_acc) : nullptr, g.T * g.D, v0 > 0, meta}, p.h, st);
            if (e != hipSuccess) return e;
        }
        if (db) {
            hipLaunchKernelGGL(bias_kernel<T>, dim3(cdiv(n, 64)), dim3(256), 0, st, meta, (const char *)G, ld_g, (int)n, db + v0);
            if ((e = hipGetLastError()) != hipSuccess) return e;
        }
    }
    if (dH && sums) {
        hipLaunchKernelGGL(finish_rows_kernel<T>, dim3((unsigned)g.T, cdiv(g.D, 1024)), dim3(256), 0, st, meta, (const float *)(ws + p.o_acc), g.T * g.D,
                           p.h.slices, (int)g.D, dH);
        e = hipGetLastError();
    }
    return e;
}

} // namespace

hipError_t launch_loss_fwd(const LossGeom &g, const LossPlan &p, const void *H, const void *W, const void *b, const int64_t *labels,
                           float *loss, float *lse, void *ws, hipStream_t st)
{
    if (g.dtype == CAC_F32) return forward(g, p, (const float *)H, (const float *)W, (const float *)b, labels, loss, lse, (char *)ws, st);
    return forward(g, p, (const bf16_t *)H, (const bf16_t *)W, (const bf16_t *)b, labels, loss, lse, (char *)ws, st);
}

hipError_t launch_loss_bwd(const LossGeom &g, const LossPlan &p, const void *H, const void *W, const void *b, const int64_t *labels,
                           const float *lse, const float *gloss, void *dH, void *dW, void *db, void *ws, hipStream_t st)
{
    if (g.dtype == CAC_F32)
        return backward(g, p, (const float *)H, (const float *)W, (const float *)b, labels, lse, gloss, (float *)dH, (float *)dW, (float *)db,
                        (char *)ws, st);
    return backward(g, p, (const bf16_t *)H, (const bf16_t *)W, (const bf16_t *)b, labels, lse, gloss, (bf16_t *)dH, (bf16_t *)dW, (bf16_t *)db,
                    (char *)ws, st);
}

} // namespace cac
