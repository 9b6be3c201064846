// A dense layer with its ending, Y = R + alpha * drop(act(u)), u = X W^T + b, and its gradients:
//   dU = drop(dY) act'(u),  dX = f dU W,  dW = f dU^T X,  db = f sum dU,  f = alpha over the probability of being kept.
// Products by matrix instructions (mm_core.h); a product's ending runs where its sums lie. What act' needs of u is not kept but formed
// again, so that the backward pass is three products; without act it is two.
//   - bfloat16: dU is rounded once, as an operand has to be; f, which is no power of two, is left out of it and multiplied into the sums, so that without
//     act dU is dY's bits. db is summed from dU before it is rounded.
//   - float: by the float instruction, operands as they lie (a matrix of any scale, infinities and NaN as float arithmetic has them).
// Sums are of 32 bits.
#include <algorithm>

#include "block.h"
#include "mm_core.h"

namespace cac {
namespace dense {
using namespace mm;

constexpr float kLog2e = 1.44269504088896340736f;

// Phi(u) = erfc(-u / sqrt 2) / 2 and exp(-u^2 / 2). For u < 0, Phi = exp(-u^2 / 2) t P(t) with t = 1 / (1 + 0.45 |u| / sqrt 2): P is a least-squares
// polynomial of erfcx(z) / (2 t), reweighted until its relative error was level; with the coefficients as they stand it is below 6e-8.  In float Phi is off by 1e-7 of
// itself in the mean down to u = -2.  Below, the exponential's argument, rounded to 24 bits of u^2 / 2, makes that grow with u^2: 2.5e-7 at -4, 5.9e-7 at -6, 1.7e-6 at -10,
// 2.3e-6 (at most 7.5e-6) at -12, where Phi is 2e-33.
__device__ __forceinline__ float normal_cdf(float u, float *bell)
{
    const float t = __builtin_amdgcn_rcpf(fmaf(0.31819805153394637f, fabsf(u), 1.f)); // 0.45 / sqrt 2
    *bell = __builtin_amdgcn_exp2f(u * u * (-0.5f * kLog2e));
    float p = -0.020695475861430168f;
    p = fmaf(p, t, 0.09534360468387604f);
    p = fmaf(p, t, -0.15029062f);
    p = fmaf(p, t, 0.07119989395141602f);
    p = fmaf(p, t, -0.011178647167980671f);
    p = fmaf(p, t, 0.05997511371970177f);
    p = fmaf(p, t, 0.08762608468532562f);
    p = fmaf(p, t, 0.11413581669330597f);
    p = fmaf(p, t, 0.12694157660007477f);
    p = fmaf(p, t, 0.12694266438484192f);
    const float below = p * t * *bell;
    return u < 0.f ? below : 1.f - below;
}
template <int ACT> __device__ __forceinline__ float activation(float u)
{
    float bell;
    if (ACT == CAC_ACT_RELU) return u <= 0.f ? 0.f : u; // (NaN stays NaN)
    if (ACT == CAC_ACT_GELU) return u * normal_cdf(u, &bell);
    if (ACT == CAC_ACT_SILU) return u * __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(-kLog2e * u));
    return u;
}
template <int ACT> __device__ __forceinline__ float slope(float u)
{
    if (ACT == CAC_ACT_RELU) return u > 0.f ? 1.f : 0.f;
    if (ACT == CAC_ACT_GELU) {
        float bell;
        const float cdf = normal_cdf(u, &bell);
        return fmaf(u * bell, 0.3989422804014327f, cdf); // 1 / sqrt(2 pi)
    }
    if (ACT == CAC_ACT_SILU) {
        const float s = __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(-kLog2e * u));
        return s * fmaf(u, 1.f - s, 1.f);
    }
    return 1.f;
}

// 256 x 256 with the loads between the products: a pass of 64 terms takes 1.56 us then (1.37 PFLOP/s; 1.62 with the loads together), and what comes before
// and after a tile's passes 14 us, of which 7 are 33 MB on their way to memory from all tiles at once.  Four waves of 128 x 128 (half the LDS
// reads) take 1.64 us a pass and twice as long at a tile's end; passes of 32 terms four or five deep, 256 x 128 and 128 x 128 two to a compute unit are slower too
// (8192 x 2048 x 8192: 257 us; 396, 276, 311 and 324).
typedef Shape<2, 4, 4, 2, 128, 2, 1, true> Large;

template <class P, Lay LA, Lay LB, class Epi>
hipError_t launch_tiles(const Params &p, const typename Epi::Params &e, TileChoice c, hipStream_t st)
{
    if constexpr (P::kRaw) {
        if constexpr (LA == Lay::kAlong)
            if (c.shape == kLow) return launch_shape<P, LA, LB, Low, Epi>(p, e, c.slices, st);
    } else {
        if (c.shape == kBig) return launch_shape<P, LA, LB, Large, Epi>(p, e, c.slices, st);
        if (c.shape == kMiddle) return launch_shape<P, LA, LB, Middle, Epi>(p, e, c.slices, st);
    }
    return launch_shape<P, LA, LB, Small, Epi>(p, e, c.slices, st);
}

// What becomes of a product's sums, or of the sums of its slices.
enum Kind {
    kForward, // R + scale drop(act(sum + b))
    kSlope,   // drop(dY) act'(sum + b), and its sums over rows
    kScaled,  // scale * sum
    kSums,    // a slice's sums as they are
};
struct Tail {
    Kind kind;
    int act, N;         // columns
    const void *b;      // [N], or null
    const void *other;  // R (or null), dY
    long ld_other;
    void *out;
    long ld_out;
    int cols_out;       // N, or up to where a row is padded with zeros
    float *columns;     // kSlope: [parts][N], or null
    float scale;
    Drop d;
    int across;         // groups of eight of a row of the mask
};

// ---- four neighbours of a row, which may start anywhere
template <typename T> struct Quad;
template <> struct Quad<float> {
    typedef uint32_t V __attribute__((ext_vector_type(4)));
    typedef V Any __attribute__((aligned(4)));
    V a;
    __device__ __forceinline__ void read(const float *p) { a = *(const Any *)p; }
    __device__ __forceinline__ void write(float *p) const { *(Any *)p = a; }
    __device__ __forceinline__ void get(float (&v)[4]) const
    {
#pragma unroll
        for (int k = 0; k < 4; ++k) v[k] = __uint_as_float(a[k]);
    }
    __device__ __forceinline__ void set(const float (&v)[4])
    {
#pragma unroll
        for (int k = 0; k < 4; ++k) a[k] = __float_as_uint(v[k]);
    }
};
template <> struct Quad<bf16_t> {
    typedef uint32_t V __attribute__((ext_vector_type(2)));
    typedef V Any __attribute__((aligned(2)));
    V a;
    __device__ __forceinline__ void read(const bf16_t *p) { a = *(const Any *)p; }
    __device__ __forceinline__ void write(bf16_t *p) const { *(Any *)p = a; }
    __device__ __forceinline__ void get(float (&v)[4]) const
    {
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            v[2 * k] = __uint_as_float(a[k] << 16);
            v[2 * k + 1] = __uint_as_float(a[k] & 0xffff0000u);
        }
    }
    __device__ __forceinline__ void set(const float (&v)[4])
    {
        a[0] = f32x2_to_bf16x2(v[0], v[1]);
        a[1] = f32x2_to_bf16x2(v[2], v[3]);
    }
};
// from column n on; zeros past N
template <typename T> __device__ __forceinline__ Quad<T> read_quad(const T *p, int n, int N)
{
    Quad<T> q;
    if (n + 4 <= N) {
        q.read(p);
        return q;
    }
    float v[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) v[k] = n + k < N ? Elem<T>::load(p + k) : 0.f;
    q.set(v);
    return q;
}
template <typename T> __device__ __forceinline__ void write_quad(T *p, int n, int N, const float (&v)[4])
{
    if (n + 4 <= N) {
        Quad<T> q;
        q.set(v);
        q.write(p);
        return;
    }
#pragma unroll
    for (int k = 0; k < 4; ++k)
        if (n + k < N) Elem<T>::store(p + k, v[k]);
}

// Four neighbours from column n on; `words` are their 64 random bits, `o` R's or dY's; `v` comes as sums and goes as what is written.
template <Kind KIND, int ACT> __device__ __forceinline__ void finish_four(const Tail &t, int n, const float (&b)[4], const float (&o)[4], const uint32_t (&words)[2], float (&v)[4])
{
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        if (KIND == kScaled) {
            v[k] *= t.scale;
        } else if (KIND == kForward) {
            const float y = t.scale * activation<ACT>(v[k] + b[k]);
            v[k] = o[k] + (!t.d.limit || drop_keeps(words[k >> 1], k & 1, t.d.limit) ? y : 0.f);
        } else if (KIND == kSlope) {
            const float g = ACT == CAC_ACT_NONE ? o[k] : o[k] * slope<ACT>(v[k] + b[k]);
            v[k] = (!t.d.limit || drop_keeps(words[k >> 1], k & 1, t.d.limit)) && n + k < t.N ? g : 0.f;
        }
    }
}

// fn(kind, act) of a tail's, as constants: asked for at every four they were branches that took 25 us of a tile
template <bool PLAIN, class Fn> __device__ __forceinline__ void with_kind(const Tail &t, Fn fn)
{
    auto acts = [&](auto kind) {
        if (t.act == CAC_ACT_GELU) fn(kind, std::integral_constant<int, CAC_ACT_GELU>());
        else if (t.act == CAC_ACT_SILU) fn(kind, std::integral_constant<int, CAC_ACT_SILU>());
        else if (t.act == CAC_ACT_RELU) fn(kind, std::integral_constant<int, CAC_ACT_RELU>());
        else fn(kind, std::integral_constant<int, CAC_ACT_NONE>());
    };
    typedef std::integral_constant<int, CAC_ACT_NONE> None;
    if (t.kind == kSums) fn(std::integral_constant<Kind, kSums>(), None());
    else if constexpr (PLAIN) fn(std::integral_constant<Kind, kScaled>(), None());
    else if (t.kind == kForward) acts(std::integral_constant<Kind, kForward>());
    else acts(std::integral_constant<Kind, kSlope>());
}

// The other lane of a pair's.
__device__ __forceinline__ uint32_t from_neighbour(uint32_t x) { return __builtin_amdgcn_update_dpp(0, x, 0xB1, 0xf, 0xf, true); }

// A product with its tail, or its slices' sums.  They go through a wave's LDS, 32 rows at a time: a lane then has four neighbours in the same
// columns of every row that it comes to, and two lanes a group of the mask, of which each forms one in two.  R (dY) of 32 rows is on its way while the
// 32 before are dealt with (of 64: 318 us where 32 take 296, 8192 x 2048 x 8192 gelu).  PLAIN: no more than a factor.
template <class T, bool PLAIN> struct Ended : Ending {
    struct Params {
        Tail t;
        float *sums; // [slice][M][N]: no tail yet
        long slice_stride;
    };
    template <int MI, int NI> static __device__ __forceinline__ void run(const Params &e, const f32x16 (&acc)[MI][NI], const Place &p)
    {
        with_kind<PLAIN>(e.t, [&](auto kind, auto act) { rows<decltype(kind)::value, decltype(act)::value, MI, NI>(e, acc, p); });
    }
    template <Kind KIND, int ACT, int MI, int NI> static __device__ __forceinline__ void rows(const Params &e, const f32x16 (&acc)[MI][NI], const Place &p)
    {
        typedef RowBlock<Fmt::kF32, NI> Block;
        constexpr int kLanes = 8 * NI, kRows = 64 / kLanes, kTurns = 32 / kRows; // lanes to a row, rows at once, turns to 32
        constexpr bool kOther = KIND == kForward || KIND == kSlope;
        const Tail &t = e.t;
        const int n = p.n0 + p.lane % kLanes * 4, row0 = p.lane / kLanes;
        float b[4] = {0.f, 0.f, 0.f, 0.f}, columns[4] = {0.f, 0.f, 0.f, 0.f};
        const bool other = kOther && t.other && n < t.N;
        if (kOther && t.b && n < t.N) read_quad((const T *)t.b + n, n, t.N).get(b);
        const DropKey key = drop_key(t.d);
        Quad<T> o[kTurns];
        auto ask = [&](int m0) {
#pragma unroll
            for (int c = 0; c < kTurns; ++c) {
                const int m = m0 + c * kRows + row0;
                if (other && m < p.M) o[c] = read_quad((const T *)t.other + (long)m * t.ld_other + n, n, t.N);
            }
        };
        const float zero[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int c = 0; c < kTurns; ++c) o[c].set(zero);
        if (kOther) ask(p.m0);
#pragma unroll
        for (int i = 0; i < MI; ++i) {
            const int m0 = p.m0 + i * 32;
#pragma unroll
            for (int j = 0; j < NI; ++j)
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    float v[4];
#pragma unroll
                    for (int k = 0; k < 4; ++k) v[k] = acc[i][j][q * 4 + k];
                    Block::put(p.lds, p.lane, j, q, v);
                }
            asm volatile("" ::: "memory"); // (a wave's LDS accesses are in order; other lanes' stores are read here)
            __builtin_amdgcn_wave_barrier();
            f32x4 x[kTurns];
            Quad<T> was[kTurns];
#pragma unroll
            for (int c = 0; c < kTurns; ++c) {
                x[c] = *(const f32x4 *)(p.lds + (c * kRows + row0) * Block::kPitch + p.lane % kLanes * 16);
                was[c] = o[c];
            }
            asm volatile("" ::: "memory");
            __builtin_amdgcn_wave_barrier();
            if (kOther && i + 1 < MI) ask(m0 + 32);
#pragma unroll
            for (int c = 0; c < kTurns; c += 2) {
                uint32_t words[2][2] = {{0, 0}, {0, 0}};
                if (kOther && t.d.limit) {
                    const bool odd = p.lane & 1;
                    const Bits128 w = drop_bits(key, t.d.site, (uint64_t)(m0 + (c + odd) * kRows + row0) * t.across + (n >> 3));
                    const uint32_t r0 = from_neighbour(odd ? w.w[0] : w.w[2]), r1 = from_neighbour(odd ? w.w[1] : w.w[3]);
                    words[0][0] = odd ? r0 : w.w[0], words[0][1] = odd ? r1 : w.w[1];
                    words[1][0] = odd ? w.w[2] : r0, words[1][1] = odd ? w.w[3] : r1;
                }
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const int m = m0 + (c + h) * kRows + row0;
                    float v[4] = {x[c + h][0], x[c + h][1], x[c + h][2], x[c + h][3]}, from[4];
                    was[c + h].get(from);
                    finish_four<KIND, ACT>(t, n, b, from, words[h], v);
                    if (m >= p.M || n >= t.cols_out) continue;
                    if (KIND == kSums) {
                        write_quad(e.sums + p.slice * e.slice_stride + (long)m * p.N + n, n, p.N, v);
                        continue;
                    }
                    if (t.out) write_quad((T *)t.out + (long)m * t.ld_out + n, n, t.cols_out, v);
                    if (KIND == kSlope) {
#pragma unroll
                        for (int k = 0; k < 4; ++k) columns[k] += v[k];
                    }
                }
            }
        }
        if (KIND != kSlope || !t.columns) return;
#pragma unroll
        for (int k = 0; k < 4; ++k)
#pragma unroll
            for (int s = kLanes; s < 64; s *= 2) columns[k] += __shfl_xor(columns[k], s, 64);
        if (p.lane < kLanes && p.m0 < p.M && n < t.N) write_quad(t.columns + (long)(p.m0 / (32 * MI)) * t.N + n, n, t.N, columns);
    }
};

// A tail without a product before it: the slices' sums joined (slices > 0), or dY alone (8192 x 2048 bfloat16 with dropout 20 to 25 us).  A thread has eight neighbours of every eighth row of
// its block's.
struct Join {
    Tail t;
    const float *sums;
    long slice_stride;
    int slices, rows_per_block;
    long M;
};
template <typename T, Kind KIND, int ACT> __device__ __forceinline__ void join_rows_of(const Join &p, float (*red)[256])
{
    const Tail &t = p.t;
    const int col = threadIdx.x & 31, turn = threadIdx.x >> 5, n = blockIdx.y * 256 + col * 8;
    const long m1 = min(p.M, (long)(blockIdx.x + 1) * p.rows_per_block);
    const DropKey key = drop_key(t.d);
    float b[2][4], columns[2][4] = {};
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int k = 0; k < 4; ++k) b[h][k] = t.b && n + h * 4 + k < t.N ? Elem<T>::load((const T *)t.b + n + h * 4 + k) : 0.f;
    if (n < t.cols_out) {
        Eight<T> ahead[2]; // R's or dY's of this row and the next
        ahead[0].clear();
        ahead[1].clear();
        const long m0 = (long)blockIdx.x * p.rows_per_block + turn;
        auto ask = [&](long m, Eight<T> &o) {
            if (KIND != kScaled && t.other && m < m1 && n < t.N) o = read_eight((const T *)t.other + m * t.ld_other, n, t.N);
        };
        ask(m0, ahead[0]);
        ask(m0 + 8, ahead[1]);
        for (long m = m0; m < m1; m += 8) {
            float from[8], v[8] = {};
            ahead[0].get(from);
            ahead[0] = ahead[1];
            ask(m + 16, ahead[1]);
            for (int k0 = 0; k0 < p.slices; k0 += 8) { // eight slices on their way at a time
                Eight<float> y[8];
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                    y[k].clear();
                    if (k0 + k < p.slices && n < t.N) y[k] = read_eight(p.sums + (k0 + k) * p.slice_stride + m * t.N, n, t.N);
                }
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                    float z[8];
                    y[k].get(z);
#pragma unroll
                    for (int e = 0; e < 8; ++e) v[e] += z[e];
                }
            }
            Bits128 w = {{0, 0, 0, 0}};
            if (KIND != kScaled && t.d.limit) w = drop_bits(key, t.d.site, (uint64_t)m * t.across + (n >> 3));
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const uint32_t words[2] = {w.w[2 * h], w.w[2 * h + 1]};
                float four[4] = {v[4 * h], v[4 * h + 1], v[4 * h + 2], v[4 * h + 3]};
                const float other[4] = {from[4 * h], from[4 * h + 1], from[4 * h + 2], from[4 * h + 3]};
                finish_four<KIND, ACT>(t, n + h * 4, b[h], other, words, four);
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    v[4 * h + k] = four[k];
                    columns[h][k] += four[k];
                }
            }
            if (t.out) write_eight((T *)t.out + m * t.ld_out, n, t.cols_out, v);
        }
    }
    if (KIND != kSlope || !t.columns) return;
#pragma unroll
    for (int e = 0; e < 8; ++e) red[turn][col * 8 + e] = columns[e >> 2][e & 3];
    __syncthreads();
    const int c = threadIdx.x;
    float s = 0.f;
    for (int k = 0; k < 8; ++k) s += red[k][c];
    if ((int)(blockIdx.y * 256) + c < t.N) t.columns[(long)blockIdx.x * t.N + blockIdx.y * 256 + c] = s;
}
struct Joins { Join j[2]; };
template <typename T> __global__ void __launch_bounds__(256) join_kernel(const Joins both)
{
    __shared__ float red[8][256];
    const Join &p = both.j[blockIdx.z];
    if ((long)blockIdx.x * p.rows_per_block >= p.M || (int)blockIdx.y * 256 >= p.t.cols_out) return;
    if (p.t.kind == kScaled) join_rows_of<T, kScaled, CAC_ACT_NONE>(p, red);
    else with_kind<false>(p.t, [&](auto kind, auto act) { join_rows_of<T, decltype(kind)::value, decltype(act)::value>(p, red); });
}

// ---- Few rows (up to 64): a workgroup has 16 features of all of them, and reads its rows of W once, as they lie, whatever they start on.  Its waves share the
// terms out, four steps of 32 (float: 16) at a time and wave; fragments come straight from memory, since a wave has no use for another's, and the waves' sums are
// joined in LDS, so that there is one launch.  bfloat16 with bias and gelu, weights that no cache holds, us in a graph (in brackets: as tiles, with a join or copy): bound by memory where weights
// are many, 1 x 8192 x 8192 30.0 (38.3) and 1 x 4096 x 4096 9.9 (15.3), 4.5 to 4.9 TB/s behind the launch's 2.6 us; by what a compute unit takes in, 31 to 36 KB a us, where features are few, 1 x 8192 x 512 11.6
// (11.6) and 16 x 8192 x 512 17.1 (12.5); by the launch where there is little, 1 x 512 x 2048 3.5 (5.8).  1 x 1001 x 2047 5.7 (15.1 with a copy of its odd rows).
struct Few {
    Tail t;
    const void *X, *W;
    long ld_x, ld_w;
    int T, K;
    void *db;       // kSlope: of T's type, times `factor`, or null
    float factor;
};
// a step's terms of one row: 8 (float: 4) to a lane
template <typename T> struct Terms;
template <> struct Terms<bf16_t> {
    static constexpr int kLane = 8, kStep = 32;
    Eight<bf16_t> v;
    __device__ __forceinline__ void clear() { v.clear(); }
    template <bool WHOLE> __device__ __forceinline__ void read(const bf16_t *row, int k, int K) { v = read_eight<WHOLE>(row, k, K); }
    static __device__ __forceinline__ f32x4 product(const Terms &a, const Terms &b, f32x4 c)
    {
        union { whole16 u; bf16x8 h; } x, y;
        x.u = a.v.a;
        y.u = b.v.a;
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(x.h, y.h, c, 0, 0, 0);
    }
};
template <> struct Terms<float> {
    static constexpr int kLane = 4, kStep = 16;
    Quad<float> v;
    __device__ __forceinline__ void clear() { v.a = Quad<float>::V{0, 0, 0, 0}; }
    template <bool WHOLE> __device__ __forceinline__ void read(const float *row, int k, int K)
    {
        if (WHOLE) v.read(row + k);
        else v = read_quad(row + k, k, K);
    }
    static __device__ __forceinline__ f32x4 product(const Terms &a, const Terms &b, f32x4 c)
    {
#pragma unroll
        for (int e = 0; e < 4; ++e) c = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(a.v.a[e]), __uint_as_float(b.v.a[e]), c, 0, 0, 0);
        return c;
    }
};
// TB: sixteens of rows.  WHOLE: rows of whole lane's terms
template <typename T, int TB, int WAVES, bool WHOLE> __global__ void __launch_bounds__(64 * WAVES) few_kernel(const Few p)
{
    typedef Terms<T> Part;
    constexpr int kAhead = 4; // steps on their way at a time
    __shared__ f32x4 red[WAVES][TB][64];
    __shared__ float db[TB][16];
    const Tail &t = p.t;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), n0 = blockIdx.x * 16, steps = (p.K + Part::kStep - 1) / Part::kStep;
    const T *w = (const T *)p.W + (long)min(n0 + (lane & 15), t.N - 1) * p.ld_w; // (what is past the last feature is not stored)
    const T *x[TB];
    bool row[TB];
#pragma unroll
    for (int i = 0; i < TB; ++i) {
        row[i] = i * 16 + (lane & 15) < p.T;
        x[i] = (const T *)p.X + (long)(row[i] ? i * 16 + (lane & 15) : 0) * p.ld_x;
    }
    const int k0 = (lane >> 4) * Part::kLane;
    struct Steps { Part a[kAhead], b[TB][kAhead]; } one, two;
    auto ask = [&](Steps &q, int s) {
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            const int k = (s + u) * Part::kStep + k0;
            q.a[u].clear();
            if (k < p.K) q.a[u].template read<WHOLE>(w, k, p.K);
#pragma unroll
            for (int i = 0; i < TB; ++i) {
                q.b[i][u].clear();
                if (k < p.K && row[i]) q.b[i][u].template read<WHOLE>(x[i], k, p.K);
            }
        }
    };
    f32x4 acc[TB];
#pragma unroll
    for (int i = 0; i < TB; ++i) acc[i] = f32x4{0.f, 0.f, 0.f, 0.f};
    auto multiply = [&](const Steps &q) {
#pragma unroll
        for (int u = 0; u < kAhead; ++u)
#pragma unroll
            for (int i = 0; i < TB; ++i) acc[i] = Part::product(q.a[u], q.b[i][u], acc[i]);
    };
    constexpr int kStride = WAVES * kAhead;
    ask(one, wave * kAhead);
    for (int s = wave * kAhead; s < steps; s += 2 * kStride) {
        ask(two, s + kStride); // (zeros behind the last)
        multiply(one);
        if (s + 2 * kStride < steps) ask(one, s + 2 * kStride);
        multiply(two);
    }
#pragma unroll
    for (int i = 0; i < TB; ++i) red[wave][i][lane] = acc[i];
    __syncthreads();
    // a wave's 16 rows by 16 features: a lane has four neighbours of a row
    const int i = wave, m = i * 16 + (lane & 15), n = n0 + (lane >> 4) * 4;
    float columns[4] = {0.f, 0.f, 0.f, 0.f};
    if (i < TB) {
        f32x4 sum = red[0][i][lane];
        for (int k = 1; k < WAVES; ++k) sum += red[k][i][lane];
        float v[4] = {sum[0], sum[1], sum[2], sum[3]}, bias[4] = {0.f, 0.f, 0.f, 0.f}, o[4] = {0.f, 0.f, 0.f, 0.f};
        const bool there = m < p.T && n < t.cols_out;
        if (t.b && n < t.N) read_quad((const T *)t.b + n, n, t.N).get(bias);
        if (t.other && there && n < t.N) read_quad((const T *)t.other + (long)m * t.ld_other + n, n, t.N).get(o);
        uint32_t words[2] = {0, 0};
        if (t.d.limit) {
            const Bits128 r = drop_bits(drop_key(t.d), t.d.site, (uint64_t)m * t.across + (n >> 3));
            words[0] = n & 4 ? r.w[2] : r.w[0];
            words[1] = n & 4 ? r.w[3] : r.w[1];
        }
        with_kind<false>(t, [&](auto kind, auto act) { finish_four<decltype(kind)::value, decltype(act)::value>(t, n, bias, o, words, v); });
        if (there) {
            if (t.out) write_quad((T *)t.out + (long)m * t.ld_out + n, n, t.cols_out, v);
#pragma unroll
            for (int k = 0; k < 4; ++k) columns[k] = v[k];
        }
        if (p.db) { // over 16 rows: lanes of the same features
#pragma unroll
            for (int k = 0; k < 4; ++k) {
#pragma unroll
                for (int s = 1; s < 16; s *= 2) columns[k] += __shfl_xor(columns[k], s, 64);
            }
            if ((lane & 15) == 0)
#pragma unroll
                for (int k = 0; k < 4; ++k) db[i][(lane >> 4) * 4 + k] = columns[k];
        }
    }
    if (!p.db) return;
    __syncthreads();
    if (threadIdx.x < 16 && n0 + (int)threadIdx.x < t.N) {
        float s = 0.f;
#pragma unroll
        for (int k = 0; k < TB; ++k) s += db[k][threadIdx.x];
        Elem<T>::store((T *)p.db + n0 + threadIdx.x, s * p.factor);
    }
}

// ---- db from the parts' sums: a block takes 64 columns, and every sixteenth part at a time, however many waves it has, so that the order is one.
struct Bias {
    const float *part;
    int parts, N;
    float scale;
    void *db;
};
template <typename T, int WAVES> __device__ __forceinline__ void bias_sums(const Bias &p, int block, float (*red)[64])
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, n = block * 64 + lane;
    for (int q = wave; q < 16; q += WAVES) {
        float s = 0.f;
        if (n < p.N) {
            const float *x = p.part + n;
            int r = q;
            for (; r + 7 * 16 < p.parts; r += 8 * 16) { // eight on their way at a time
                float y[8];
#pragma unroll
                for (int k = 0; k < 8; ++k) y[k] = x[(long)(r + k * 16) * p.N];
#pragma unroll
                for (int k = 0; k < 8; ++k) s += y[k];
            }
            for (; r < p.parts; r += 16) s += x[(long)r * p.N];
        }
        red[q][lane] = s;
    }
    __syncthreads();
    if (wave || n >= p.N) return;
    float s = red[0][lane];
    for (int q = 1; q < 16; ++q) s += red[q][lane];
    Elem<T>::store((T *)p.db + n, s * p.scale);
}
template <typename T> __global__ void __launch_bounds__(1024) bias_join_kernel(const Bias p)
{
    __shared__ float red[16][64];
    bias_sums<T, 16>(p, blockIdx.x, red);
}

// ---- dX, dW and db in one launch: the products' workgroups fill the compute units together, and the longer sums begin first.  300 x 300 x 300 bfloat16 16.2 to
// 10.2 us, 1531 x 1001 x 515 float 95 to 81, 4096 x 2048 x 8192 gelu 412 to 389.
template <typename T> struct Pair {
    Params x, w;
    typename Ended<T, true>::Params ex, ew;
    Bias b;
    unsigned blocks_first, blocks_second;
    bool x_first;
};
template <class P, class S, typename T> __global__ void __launch_bounds__(S::kThreads, S::kPerSimd) pair_kernel(const Pair<T> p)
{
    extern __shared__ __align__(1024) unsigned char smem[];
    unsigned block = blockIdx.x;
    const bool first = block < p.blocks_first;
    if (!first) block -= p.blocks_first;
    if (!first && block >= p.blocks_second) {
        bias_sums<T, S::kWaves>(p.b, block - p.blocks_second, (float(*)[64])smem);
    } else if (first == p.x_first) {
        mm_tile<P, Lay::kAlong, Lay::kDown, S, Ended<T, true>>(p.x, p.ex, block, smem);
    } else {
        mm_tile<P, Lay::kDown, Lay::kDown, S, Ended<T, true>>(p.w, p.ew, block, smem);
    }
}
template <class P, class S, typename T> hipError_t launch_pair(Pair<T> p, TileChoice cx, TileChoice cw, hipStream_t st)
{
    static const hipError_t attr = hipFuncSetAttribute(reinterpret_cast<const void *>(pair_kernel<P, S, T>), hipFuncAttributeMaxDynamicSharedMemorySize, S::kLds);
    if (attr != hipSuccess) return attr;
    const unsigned bx = place_tiles<S>(&p.x, false, cx.slices, kPass<P, S::R>), bw = place_tiles<S>(&p.w, false, cw.slices, kPass<P, S::R>);
    p.x_first = p.x.kt_slice >= p.w.kt_slice;
    p.blocks_first = p.x_first ? bx : bw;
    p.blocks_second = p.x_first ? bw : bx;
    const unsigned bias = p.b.db ? (unsigned)cdiv(p.b.N, 64) : 0;
    hipLaunchKernelGGL((pair_kernel<P, S, T>), dim3(bx + bw + bias), dim3(S::kThreads), S::kLds, st, p);
    return hipGetLastError();
}

// Rows of any length and stride to rows of whole units of 16 bytes, padded with zeros; both operands in one launch.
struct Pack {
    const void *from[2];
    void *to[2];
    long ld[2];
    long groups[2]; // of eight elements, of all rows; 0: not this one
    int columns;    // (both have the same)
};
template <typename T> __global__ void __launch_bounds__(256) pack_kernel(const Pack p)
{
    const int across = (p.columns + 7) / 8;
    for (long g = (long)blockIdx.x * 256 + threadIdx.x; g < p.groups[0] + p.groups[1]; g += (long)gridDim.x * 256) {
        const bool second = g >= p.groups[0];
        const long at = second ? g - p.groups[0] : g, row = at / across;
        const int n = (int)(at - row * across) * 8;
        const T *x = (const T *)(second ? p.from[1] : p.from[0]) + row * (second ? p.ld[1] : p.ld[0]);
        float v[8];
        read_eight(x, n, p.columns).get(v);
        write_eight((T *)(second ? p.to[1] : p.to[0]) + at * 8, 0, 8, v);
    }
}

} // namespace dense

using namespace dense;

// ---- host
constexpr int kFewRows = 64;

// Microseconds of M x N sums of K terms in a tile and a number of slices.  What a pass takes on a compute unit with one workgroup and with as many
// as it holds, and what comes before and after a workgroup's passes: from 8192 x 64 x 8192 to 8192 x 8192 x 2048 bfloat16 within 8 %. The slices' sums
// are written, read and joined in a launch of their own, 4 us.
struct Price { int holds; double alone, full, once, once_full; };
static Price price_of(Format f, int shape)
{
    static const Price kBf[] = {{3, 0.27, 0.72, 2.5, 4.0}, {2, 0.77, 1.06, 3.5, 7.0}, {}, {1, 1.56, 1.56, 9.0, 14.0}, {}},
                       kRawOf[] = {{3, 0.5, 1.4, 2.5, 4.0}, {}, {}, {}, {2, 0.5, 1.0, 2.5, 4.0}};
    return (f == kRaw ? kRawOf : kBf)[shape];
}
// What an ending adds to that: an activation with an exponential, dropout, and R or dY to be read.  The largest tile has nothing else to do meanwhile
// (8192 x 256 x 8192 with all three: 187 us in tiles of 256, 139 of 128, 177 of 64).
struct Extra { bool exponential, drops, other; };
static double ending_us(int shape, const Extra &x)
{
    static const double kUs[kShapes][3] = {{1.0, 0.5, 0.8}, {2.7, 1.1, 2.2}, {}, {7.5, 2.5, 12.0}, {1.0, 0.5, 0.8}};
    return x.exponential * kUs[shape][0] + x.drops * kUs[shape][1] + x.other * kUs[shape][2];
}
static double tiles_us(Format f, int shape, long M, long N, long K, int slices, const Extra &x)
{
    Price p = price_of(f, shape);
    const double ending = slices > 1 ? 0.0 : ending_us(shape, x);
    p.once += ending;
    p.once_full += ending;
    const double n = cdiv(cdiv(K, kTerms[f]), slices);
    const long wgs = tiles_of(shape, M, N, false) * slices, round = 256L * p.holds, rest = wgs % round;
    double us = (wgs / round) * (p.full * n + p.once_full);
    if (rest) {
        const double share = rest <= 256 ? rest / 256.0 * (p.holds == 1) : (rest - 256.0) / (round - 256);
        const double pass = rest <= 256 ? p.alone : p.alone + share * (p.full - p.alone);
        us += pass * n + p.once + share * (p.once_full - p.once);
    }
    if (slices > 1) us += 4.0 + 3.2e-6 * slices * M * N;
    return us;
}
// The cheapest; false: too many tiles for one grid.  DOWN: a's terms run down memory, which tiles of 32 rows have no layout for.
static bool choose_tiles(Format f, long M, long N, long K, bool down, const Extra &x, TileChoice *c, double *least)
{
    *least = 1e30;
    for (int shape = 0; shape < kShapes; ++shape) {
        if (f == kRaw ? shape != kSmall && shape != kLow : shape == kLow || shape == kWide) continue;
        if (f == kRaw && (shape == kLow) != (M <= 32 && !down)) continue;
        const long tiles = tiles_of(shape, M, N, false);
        for (int slices = 1; slices <= 64; slices += slices < 4 ? 1 : slices / 4 * 2) {
            if (slices > 1 && (cdiv(K, kTerms[f]) / slices < 4 || tiles * slices > 2048)) break;
            if (!fits_grid(shape, tiles * slices)) break;
            const double us = tiles_us(f, shape, M, N, K, slices, x);
            if (us < *least) {
                *least = us;
                *c = TileChoice{shape, slices};
            }
        }
    }
    return *least < 1e30;
}
// dX and dW in one launch, tiles of one kind: what all workgroups take of the compute units, or the longest of them.
struct PairChoice { TileChoice x, w; double us; };
static PairChoice choose_pair(Format f, const LinearGeom &g)
{
    PairChoice best = {{}, {}, 1e30};
    for (int shape : {kSmall, kMiddle, kBig}) {
        if (f == kRaw && shape != kSmall) continue;
        const Price p = price_of(f, shape);
        const long tx = tiles_of(shape, g.T, g.D, false), tw = tiles_of(shape, g.N, g.D, false);
        const int nx = cdiv(g.N, kTerms[f]), nw = cdiv(g.T, kTerms[f]);
        for (int sx = 1; sx <= 32; sx *= 2)
            for (int sw = 1; sw <= 32; sw *= 2) {
                if ((sx > 1 && (nx / sx < 4 || tx * sx > 2048)) || (sw > 1 && (nw / sw < 4 || tw * sw > 2048))) continue;
                const long wgs = tx * sx + tw * sw;
                if (!fits_grid(shape, wgs + cdiv(g.N, 64) + 16)) continue;
                // with fewer workgroups than the card holds a pass takes less
                const double fill = std::min(1.0, std::max(0.0, (wgs / 256.0 - 1) / std::max(1, p.holds - 1))), pass = p.alone + fill * (p.full - p.alone);
                const double once = p.holds == 1 ? p.once_full : p.once + fill * (p.once_full - p.once);
                const double cx = cdiv(nx, sx) * pass + once, cw = cdiv(nw, sw) * pass + once;
                double us = std::max(std::max(cx, cw), (tx * sx * cx + tw * sw * cw) / (256.0 * p.holds));
                if (sx > 1 || sw > 1) us += 4.0 + 3.2e-6 * ((sx > 1 ? sx * g.T * g.D : 0) + (sw > 1 ? sw * g.N * g.D : 0));
                if (us < best.us) best = PairChoice{{shape, sx}, {shape, sw}, us};
            }
    }
    return best;
}
// Few rows by few_kernel, as if all that bound it were what a compute unit takes in, 35 KB a us: its features' rows of W, and X.  Of one to four rows with many weights that is
// too little (1 x 4096 x 4096 bfloat16 6.6 where it takes 9.9 us, 1 x 8192 x 8192 18.5 where 30.0), but so is what tiles are priced at there.  Of 154 layers of 1 to 64
// rows, 512 to 8192 columns and features, in either type, none goes to few_kernel that tiles are faster with; 13 go to tiles that few_kernel does up to 14 %
// (4 x 8192 x 8192 float 22 %) faster: 1 x 8192 x 2048 float 30.6 / 26.2 us, 2 x 8192 x 2048 bfloat16 15.4 / 13.8, 16 x 4096 x 1024 bfloat16 11.0 / 10.0.
static double few_us(long T, long N, long K, long e) { return 2.6 + cdiv(cdiv(N, 16), 256) * (16.0 + T) * K * e / 35e3; }

static int rows_of_a_part(int shape) // of a tile, that one wave sums over
{
    static const int kRowsOf[kShapes] = {32 * Small::MI, 32 * Middle::MI, 32 * Wide::MI, 32 * Large::MI, 32 * Low::MI};
    return kRowsOf[shape];
}
static long join_rows(long M) { return M < 2048 ? 8 : 64; } // of a block of join_kernel

bool plan_linear(const LinearGeom &g, bool backward, LinearPlan *p)
{
    const Format f = g.dtype == CAC_F32 ? kRaw : kBf16;
    const long e = g.dtype == CAC_F32 ? 4 : 2, whole = 16 / e;
    auto padded = [&](long n) { return (n + 7) / 8 * 8; };
    size_t at = 0;
    auto take = [&](size_t bytes) {
        const size_t o = at;
        at += (bytes + 255) / 256 * 256;
        return o;
    };
    *p = LinearPlan{};
    p->pack_x = g.D % whole || g.ld_x % whole;
    p->pack_w = g.D % whole || g.ld_w % whole;
    p->ld_x = p->pack_x ? padded(g.D) : g.ld_x;
    p->ld_w = p->pack_w ? padded(g.D) : g.ld_w;
    p->again = backward && g.act != CAC_ACT_NONE;
    p->grad = backward && (p->again || g.drops || g.N % whole);
    p->ld_u = p->grad ? padded(g.N) : g.N;
    size_t sums = 0;
    double us;
    auto product = [&](long M, long N, long K, bool down, TileChoice *c, const Extra &x = Extra{}) {
        if (!choose_tiles(f, M, N, K, down, x, c, &us)) return false;
        if (c->slices > 1 && sums < (size_t)c->slices * M * N * 4) sums = (size_t)c->slices * M * N * 4;
        return true;
    };
    if (!backward || p->again) {
        const Extra x = {g.act == CAC_ACT_GELU || g.act == CAC_ACT_SILU, g.drops, backward}; // (a forward pass without R has the same plan as one with it)
        if (!product(g.T, g.N, g.D, false, &p->y, x)) return false;
        if ((p->pack_x || p->pack_w) && !backward) us += 4.0 + (g.T + g.N) * g.D * e * 1e-6 / 1.5;
        p->few = g.T <= kFewRows && few_us(g.T, g.N, g.D, e) < us;
        if (p->few) sums = 0;
        if (p->few && !backward) p->pack_x = p->pack_w = false;
    }
    if (p->pack_x) p->o_x = take(g.T * p->ld_x * e);
    if (p->pack_w) p->o_w = take(g.N * p->ld_w * e);
    if (backward) {
        double both = 4.0; // (a launch)
        if (!product(g.T, g.D, g.N, false, &p->dx)) return false;
        both += us;
        if (!product(g.N, g.D, g.T, true, &p->dw)) return false;
        both += us;
        const PairChoice pair = choose_pair(f, g);
        if (pair.us < both) {
            p->together = true;
            p->dx = pair.x;
            p->dw = pair.w;
        }
        p->parts = p->again && p->few ? 0 : p->again && p->y.slices == 1 ? cdiv(g.T, rows_of_a_part(p->y.shape)) : cdiv(g.T, join_rows(g.T));
        if (p->grad) p->o_u = take(g.T * p->ld_u * e);
        p->o_db = take((size_t)p->parts * g.N * 4);
    }
    p->o_sum = take(sums);
    if (p->together) {
        const size_t sx = p->dx.slices > 1 ? (size_t)p->dx.slices * g.T * g.D * 4 : 0, sw = p->dw.slices > 1 ? (size_t)p->dw.slices * g.N * g.D * 4 : 0;
        at = p->o_sum; // (the pre-activation's slices have been joined by then, and one of the two products may be asked for alone)
        take(std::max(sums, sx));
        p->o_sum2 = take(sw);
        at = std::max(at, p->o_sum + (sw + 255) / 256 * 256);
    }
    p->bytes = at;
    return true;
}

namespace {

template <typename T> struct Layer {
    static constexpr bool kFloat = sizeof(T) == 4;
    typedef typename std::conditional<kFloat, Raw, Bf16>::type P;
    const LinearGeom &g;
    const LinearPlan &p;
    const Drop &d;
    char *ws;
    hipStream_t st;
    hipError_t err = hipSuccess;

    const void *x, *w; // as they are multiplied

    void pack(const void *X, const void *W, bool need_x, bool need_w)
    {
        const bool px = p.pack_x && need_x, pw = p.pack_w && need_w;
        x = px ? ws + p.o_x : X;
        w = pw ? ws + p.o_w : W;
        if (!px && !pw) return;
        Pack a;
        a.from[0] = X, a.from[1] = W;
        a.to[0] = ws + p.o_x, a.to[1] = ws + p.o_w;
        a.ld[0] = g.ld_x, a.ld[1] = g.ld_w;
        const long across = (g.D + 7) / 8;
        a.groups[0] = px ? g.T * across : 0;
        a.groups[1] = pw ? g.N * across : 0;
        a.columns = (int)g.D;
        const long blocks = (a.groups[0] + a.groups[1] + 255) / 256;
        hipLaunchKernelGGL((pack_kernel<T>), dim3((unsigned)(blocks < 8192 ? blocks : 8192)), dim3(256), 0, st, a);
        err = hipGetLastError();
    }
    Tail tail(Kind kind, long N, void *out, long ld_out) const
    {
        Tail t = {};
        t.kind = kind;
        t.act = g.act;
        t.N = (int)N;
        t.out = out;
        t.ld_out = ld_out;
        t.cols_out = (int)N;
        t.scale = g.alpha * d.scale;
        t.across = (int)((N + 7) / 8);
        return t;
    }
    Join joined(const Tail &t, long M, int slices, size_t o_sum) const
    {
        Join j;
        j.t = t;
        j.sums = (const float *)(ws + o_sum);
        j.slice_stride = M * t.N;
        j.slices = slices;
        j.M = M;
        j.rows_per_block = (int)join_rows(M);
        return j;
    }
    void join(const Join &a, const Join *b = nullptr)
    {
        auto across = [](const Join &j) { return (unsigned)cdiv(j.M, j.rows_per_block); };
        auto down = [](const Join &j) { return (unsigned)cdiv(j.t.cols_out, 256); };
        const Joins both = {{a, b ? *b : a}};
        const dim3 grid(b ? std::max(across(a), across(*b)) : across(a), b ? std::max(down(a), down(*b)) : down(a), b ? 2 : 1);
        hipLaunchKernelGGL((join_kernel<T>), grid, dim3(256), 0, st, both);
        err = hipGetLastError();
    }
    void few(const void *X, const void *W, const Tail &t, void *db)
    {
        if (err != hipSuccess) return;
        Few f;
        f.t = t;
        f.X = X;
        f.W = W;
        f.ld_x = g.ld_x;
        f.ld_w = g.ld_w;
        f.T = (int)g.T;
        f.K = (int)g.D;
        f.db = db;
        f.factor = t.scale;
        auto go = [&](auto kernel, int waves) { hipLaunchKernelGGL(kernel, dim3((unsigned)cdiv(t.cols_out, 16)), dim3(64 * waves), 0, st, f); };
        // a wave has 4 steps at a time; with more waves than that gives work to, the others only wait
        const bool wide = g.D > 4 * 4 * Terms<T>::kStep;
        auto waves = [&](auto sixteens, auto whole) {
            constexpr int kMost = decltype(sixteens)::value > 2 ? 8 : 16; // (what registers leave room for)
            if (wide) go(few_kernel<T, decltype(sixteens)::value, kMost, decltype(whole)::value>, kMost);
            else go(few_kernel<T, decltype(sixteens)::value, 4, decltype(whole)::value>, 4);
        };
        auto rows = [&](auto sixteens) {
            if (g.D % Terms<T>::kLane) waves(sixteens, std::false_type());
            else waves(sixteens, std::true_type());
        };
        if (g.T <= 16) rows(std::integral_constant<int, 1>());
        else if (g.T <= 32) rows(std::integral_constant<int, 2>());
        else rows(std::integral_constant<int, 4>());
        err = hipGetLastError();
    }
    // C = A B^T with a tail, the sums of whose slices go to o_sum
    template <class Epi> void describe(mm::Params *m, typename Epi::Params *e, const void *a, long lda, const void *b, long ldb, long M, long N, long K, TileChoice c,
                                       const Tail &t, size_t o_sum) const
    {
        *m = mm::Params{};
        m->a = a;
        m->b = b;
        m->lda = lda * sizeof(T);
        m->ldb = ldb * sizeof(T);
        m->M = (int)M;
        m->N = (int)N;
        m->K = (int)K;
        m->batch = 1;
        e->t = t;
        e->sums = c.slices > 1 ? (float *)(ws + o_sum) : nullptr;
        e->slice_stride = M * N;
        if (e->sums) {
            e->t.kind = kSums;
            e->t.cols_out = (int)N;
        }
    }
    template <Lay LA, Lay LB> void product(const void *a, long lda, const void *b, long ldb, long M, long N, long K, TileChoice c, const Tail &t)
    {
        if (err != hipSuccess) return;
        typedef Ended<T, LB == Lay::kDown> Epi;
        mm::Params m;
        typename Epi::Params e;
        describe<Epi>(&m, &e, a, lda, b, ldb, M, N, K, c, t, p.o_sum);
        err = launch_tiles<P, LA, LB, Epi>(m, e, c, st);
        if (err == hipSuccess && c.slices > 1) join(joined(t, M, c.slices, p.o_sum));
    }
    Bias bias(void *db) const { return Bias{(const float *)(ws + p.o_db), (int)p.parts, (int)g.N, g.alpha * d.scale, p.parts ? db : nullptr}; }
    void pair(const void *u, void *dX, void *dW, void *db)
    {
        if (err != hipSuccess) return;
        const Tail tx = tail(kScaled, g.D, dX, g.D), tw = tail(kScaled, g.D, dW, g.D);
        Pair<T> a = {};
        describe<Ended<T, true>>(&a.x, &a.ex, u, p.ld_u, w, p.ld_w, g.T, g.D, g.N, p.dx, tx, p.o_sum);
        describe<Ended<T, true>>(&a.w, &a.ew, u, p.ld_u, x, p.ld_x, g.N, g.D, g.T, p.dw, tw, p.o_sum2);
        a.b = bias(db);
        if constexpr (kFloat) {
            err = launch_pair<P, Small, T>(a, p.dx, p.dw, st);
        } else {
            if (p.dx.shape == kBig) err = launch_pair<P, Large, T>(a, p.dx, p.dw, st);
            else if (p.dx.shape == kMiddle) err = launch_pair<P, Middle, T>(a, p.dx, p.dw, st);
            else err = launch_pair<P, Small, T>(a, p.dx, p.dw, st);
        }
        if (err != hipSuccess) return;
        const Join jx = joined(tx, g.T, p.dx.slices, p.o_sum), jw = joined(tw, g.N, p.dw.slices, p.o_sum2);
        if (p.dx.slices > 1 && p.dw.slices > 1) join(jx, &jw);
        else if (p.dx.slices > 1) join(jx);
        else if (p.dw.slices > 1) join(jw);
    }
    hipError_t forward(const void *X, const void *W, const void *b, const void *R, void *Y)
    {
        pack(X, W, true, true);
        Tail t = tail(kForward, g.N, Y, g.N);
        t.b = b;
        t.other = R;
        t.ld_other = g.ld_r;
        t.d = d;
        if (p.few) few(X, W, t, nullptr);
        else product<Lay::kAlong, Lay::kAlong>(x, p.ld_x, w, p.ld_w, g.T, g.N, g.D, p.y, t);
        return err;
    }
    hipError_t backward(const void *X, const void *W, const void *b, const void *dY, void *dX, void *dW, void *db)
    {
        pack(X, W, dW || (p.again && !p.few), dX || (p.again && !p.few));
        const void *u = p.grad ? ws + p.o_u : dY;
        Tail t = tail(kSlope, g.N, p.grad ? ws + p.o_u : nullptr, p.ld_u);
        t.cols_out = (int)p.ld_u;
        t.b = b;
        t.other = dY;
        t.ld_other = g.N;
        t.columns = db ? (float *)(ws + p.o_db) : nullptr;
        t.d = d;
        if (p.again && p.few) few(X, W, t, db);
        else if (p.again) product<Lay::kAlong, Lay::kAlong>(x, p.ld_x, w, p.ld_w, g.T, g.N, g.D, p.y, t);
        else if (err == hipSuccess && (p.grad || db)) join(joined(t, g.T, 0, p.o_sum));
        if (dX && dW && p.together) {
            pair(u, dX, dW, db);
            return err;
        }
        if (dX) product<Lay::kAlong, Lay::kDown>(u, p.ld_u, w, p.ld_w, g.T, g.D, g.N, p.dx, tail(kScaled, g.D, dX, g.D));
        if (dW) product<Lay::kDown, Lay::kDown>(u, p.ld_u, x, p.ld_x, g.N, g.D, g.T, p.dw, tail(kScaled, g.D, dW, g.D));
        if (db && p.parts && err == hipSuccess) {
            hipLaunchKernelGGL((bias_join_kernel<T>), dim3((unsigned)cdiv(g.N, 64)), dim3(1024), 0, st, bias(db));
            err = hipGetLastError();
        }
        return err;
    }
};

} // namespace

hipError_t launch_linear_fwd(const LinearGeom &g, const LinearPlan &p, const Drop &d, const void *X, const void *W, const void *b, const void *R,
                             void *Y, void *ws, hipStream_t st)
{
    if (g.dtype == CAC_F32) return Layer<float>{g, p, d, (char *)ws, st}.forward(X, W, b, R, Y);
    return Layer<bf16_t>{g, p, d, (char *)ws, st}.forward(X, W, b, R, Y);
}

hipError_t launch_linear_bwd(const LinearGeom &g, const LinearPlan &p, const Drop &d, const void *X, const void *W, const void *b, const void *dY,
                             void *dX, void *dW, void *db, void *ws, hipStream_t st)
{
    if (g.dtype == CAC_F32) return Layer<float>{g, p, d, (char *)ws, st}.backward(X, W, b, dY, dX, dW, db);
    return Layer<bf16_t>{g, p, d, (char *)ws, st}.backward(X, W, b, dY, dX, dW, db);
}

} // namespace cac
