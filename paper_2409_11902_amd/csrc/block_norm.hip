// What stands between two blocks of a residual network:
//   forward : S = R + alpha * drop(gate * post(F)),  H = pre(S)
//   backward: dR = dS + pre'(S)^T dH,  a = alpha * drop(dR),  dF = post'(F)^T (gate * a), and the sums over rows for the gate and the
//             norms' weights.
// A norm's statistics of a row are formed from the row in registers, in the forward pass and again in the backward pass, so that neither they
// nor the normalised row nor the mask is kept: what the backward pass reads is F and S.  With xhat = (x - mean) / sqrt(var + eps), g the gradient of
// xhat:  dx = (g - mean(g) - xhat mean(g xhat)) / sqrt(var + eps), without the first two means for rms.
// Bound by memory: every row is read and written once.  A row is spread over the lanes of one to sixteen waves, eight
// neighbours to a lane (two groups of eight above 8192 columns); weights stay in registers while a workgroup goes from row to
// row, and so do the sums over rows, whose order is fixed: a workgroup's, then the workgroups'.
#include "block.h"

namespace cac {

struct NormArgs {
    NormGeom g;
    NormPlan p;
    Drop d;
    NormParams w;
    float scale;                 // alpha over the probability of being kept
    float inv_d;
    bool wide, wide_f, wide_r;   // rows of whole groups on 16 bytes: the dense ones, F's, R's
    const void *F, *R, *S_in, *dH, *dS;
    void *S, *H, *dR, *dF;
    NormGrads o;
    float *part;                 // [5][blocks][D], of the sums in NormGrads' order
};

// The sum over a wave in every lane, in one order for all of them.
__device__ __forceinline__ float wave_total(float x)
{
    auto moved = [](float v, auto ctrl) { return __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(v), decltype(ctrl)::value, 0xf, 0xf, true)); };
    x += moved(x, std::integral_constant<int, 0xB1>());  // neighbours
    x += moved(x, std::integral_constant<int, 0x4E>());  // pairs
    x += moved(x, std::integral_constant<int, 0x141>()); // fours, mirrored
    x += moved(x, std::integral_constant<int, 0x140>()); // eights, mirrored
    auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    x = __uint_as_float(r[0]) + __uint_as_float(r[1]);
    r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

// The sums of two numbers over the WPR waves of a row.  `red` holds two turns, so that one meeting is enough: a wave that writes a turn's
// numbers has met since the others read those of the turn before.
template <int WPR> struct RowSum {
    float2 *red; // [2][waves of the workgroup]
    int wave, waves, turn;
    __device__ __forceinline__ void operator()(float &a, float &b)
    {
        a = wave_total(a);
        b = wave_total(b);
        if (WPR == 1) return;
        float2 *r = red + turn * waves;
        if ((threadIdx.x & 63) == 0) r[wave] = make_float2(a, b);
        __syncthreads();
        const int first = wave / WPR * WPR;
        a = b = 0.f;
#pragma unroll
        for (int k = 0; k < WPR; ++k) {
            const float2 v = r[first + k];
            a += v.x;
            b += v.y;
        }
        turn ^= 1;
    }
};

// eight of a vector of weights, `otherwise` where there is none
__device__ __forceinline__ void eight_weights(const float *w, int n, int D, float otherwise, float (&v)[8])
{
    if (!w) {
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = otherwise;
    } else if (D % 4 == 0 && n + 8 <= D) { // (rows of the gate start on 16 bytes then)
        Eight<float> x;
        x.read(w + n);
        x.get(v);
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = n + e < D ? w[n + e] : 0.f;
    }
}

// Mean (zero for rms) and one over the spread of a row,
template <int WPR, int CH>
__device__ __forceinline__ float2 statistics(int kind, float eps, const float (&a)[CH][8], const int (&count)[CH], float inv_d, RowSum<WPR> &sum)
{
    float m = 0.f, v = 0.f, none = 0.f;
    if (kind == CAC_NORM_LAYER) {
#pragma unroll
        for (int c = 0; c < CH; ++c)
#pragma unroll
            for (int e = 0; e < 8; ++e) m += a[c][e];
        sum(m, none);
        m *= inv_d;
    }
#pragma unroll
    for (int c = 0; c < CH; ++c)
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float x = e < count[c] ? a[c][e] - m : 0.f; // (what is read past a row's end is zero, and the mean away from it)
            v += x * x;
        }
    none = 0.f;
    sum(v, none);
    return make_float2(m, 1.f / sqrtf(v * inv_d + eps));
}
// ... and of two rows with the meetings of one.
template <int WPR, int CH>
__device__ __forceinline__ void statistics2(int kind_a, float eps_a, const float (&a)[CH][8], float2 *of_a, int kind_b, float eps_b, const float (&b)[CH][8], float2 *of_b,
                                            const int (&count)[CH], float inv_d, RowSum<WPR> &sum)
{
    float ma = 0.f, mb = 0.f, va = 0.f, vb = 0.f;
    if (kind_a == CAC_NORM_LAYER || kind_b == CAC_NORM_LAYER) {
#pragma unroll
        for (int c = 0; c < CH; ++c)
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                ma += a[c][e];
                mb += b[c][e];
            }
        sum(ma, mb);
        ma = kind_a == CAC_NORM_LAYER ? ma * inv_d : 0.f;
        mb = kind_b == CAC_NORM_LAYER ? mb * inv_d : 0.f;
    }
#pragma unroll
    for (int c = 0; c < CH; ++c)
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float x = e < count[c] ? a[c][e] - ma : 0.f, y = e < count[c] ? b[c][e] - mb : 0.f;
            va += x * x;
            vb += y * y;
        }
    sum(va, vb);
    *of_a = make_float2(ma, 1.f / sqrtf(va * inv_d + eps_a));
    *of_b = make_float2(mb, 1.f / sqrtf(vb * inv_d + eps_b));
}

template <int WPR> constexpr int kFwdWaves = WPR > 4 ? WPR : 4;
template <int WPR> constexpr int kBwdWaves = WPR > 8 ? WPR : 8;

template <typename T, int WPR, int CH> __global__ void __launch_bounds__(64 * kFwdWaves<WPR>) norm_fwd_kernel(const NormArgs a)
{
    constexpr int kWaves = kFwdWaves<WPR>, kSlots = kWaves / WPR;
    __shared__ float2 red[2 * kWaves];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), slot = wave / WPR, D = (int)a.g.D;
    RowSum<WPR> sum{red, wave, kWaves, 0};
    const long r0 = blockIdx.x * a.p.rows_per_block, r1 = min(a.g.T, r0 + a.p.rows_per_block);
    int n[CH], count[CH];
#pragma unroll
    for (int c = 0; c < CH; ++c) {
        n[c] = ((c * WPR + wave % WPR) * 64 + lane) * 8;
        count[c] = min(max(D - n[c], 0), 8);
    }
    const int across = (D + 7) / 8;
    const DropKey key = drop_key(a.d);
    Eight<T> f[CH], r[CH];
    auto ask = [&](long row) {
#pragma unroll
        for (int c = 0; c < CH; ++c)
            if (count[c]) {
                f[c] = read_eight((const T *)a.F + row * a.g.ld_f, n[c], D, a.wide_f);
                if (a.R) r[c] = read_eight((const T *)a.R + row * a.g.ld_r, n[c], D, a.wide_r);
            }
    };
    const float zero[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int c = 0; c < CH; ++c) {
        f[c].set(zero);
        r[c].set(zero);
    }
    if (r0 + slot < r1) ask(r0 + slot);
    float w_post[CH][8], b_post[CH][8], w_pre[CH][8], b_pre[CH][8], gate[CH][8];
#pragma unroll
    for (int c = 0; c < CH; ++c) {
        eight_weights(a.w.w_post, n[c], D, 1.f, w_post[c]);
        eight_weights(a.w.b_post, n[c], D, 0.f, b_post[c]);
        eight_weights(a.w.w_pre, n[c], D, 1.f, w_pre[c]);
        eight_weights(a.w.b_pre, n[c], D, 0.f, b_pre[c]);
    }
    long group = -1;
    for (long base = r0; base < r1; base += kSlots) {
        const long row = base + slot;
        const bool there = row < r1;
        float v[CH][8], s[CH][8];
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            f[c].get(v[c]);
            r[c].get(s[c]);
        }
        if (row + kSlots < r1) ask(row + kSlots);
        const long here = a.g.gate_rows ? row / a.g.gate_rows : 0;
        if (here != group) {
            group = here;
#pragma unroll
            for (int c = 0; c < CH; ++c) eight_weights(a.w.gate && there ? a.w.gate + here * D : nullptr, n[c], D, 1.f, gate[c]);
        }
        if (a.g.post != CAC_NORM_NONE) {
            const float2 st = statistics<WPR, CH>(a.g.post, a.g.eps_post, v, count, a.inv_d, sum);
#pragma unroll
            for (int c = 0; c < CH; ++c)
#pragma unroll
                for (int e = 0; e < 8; ++e) v[c][e] = (v[c][e] - st.x) * st.y * w_post[c][e] + b_post[c][e];
        }
#pragma unroll
        for (int c = 0; c < CH; ++c) {
#pragma unroll
            for (int e = 0; e < 8; ++e) v[c][e] *= gate[c][e];
            drop_eight(key, a.d, (uint64_t)(row * across + (n[c] >> 3)), a.scale, v[c]);
#pragma unroll
            for (int e = 0; e < 8; ++e) s[c][e] = e < count[c] ? s[c][e] + v[c][e] : 0.f;
            if (there && count[c] && a.S) write_eight((T *)a.S + row * D, n[c], D, a.wide, s[c]);
        }
        if (!a.H) continue;
        const float2 st = statistics<WPR, CH>(a.g.pre, a.g.eps_pre, s, count, a.inv_d, sum);
#pragma unroll
        for (int c = 0; c < CH; ++c) {
#pragma unroll
            for (int e = 0; e < 8; ++e) s[c][e] = (s[c][e] - st.x) * st.y * w_pre[c][e] + b_pre[c][e];
            if (there && count[c]) write_eight((T *)a.H + row * D, n[c], D, a.wide, s[c]);
        }
    }
}

enum { kGate, kWPost, kBPost, kWPre, kBPre, kSums };

template <typename T, int WPR, int CH> __global__ void __launch_bounds__(64 * kBwdWaves<WPR>, 4) norm_bwd_kernel(const NormArgs a)
{
    constexpr int kWaves = kBwdWaves<WPR>, kSlots = kWaves / WPR, kColumns = 512 * WPR * CH;
    __shared__ float2 red[2 * kWaves];
    __shared__ float joined[kSlots > 1 ? (kSlots - 1) * kColumns : 1];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), slot = wave / WPR, D = (int)a.g.D;
    RowSum<WPR> sum{red, wave, kWaves, 0};
    int n[CH], count[CH];
#pragma unroll
    for (int c = 0; c < CH; ++c) {
        n[c] = ((c * WPR + wave % WPR) * 64 + lane) * 8;
        count[c] = min(max(D - n[c], 0), 8);
    }
    const int across = (D + 7) / 8;
    const DropKey key = drop_key(a.d);
    const bool post = a.g.post != CAC_NORM_NONE, pre = a.g.pre != CAC_NORM_NONE, gated = a.w.gate != nullptr;

    // Rows: a run of one group's, the slots taking turns; or (own_groups) every slot has whole groups to itself, this many apart.
    const long G = a.g.gate_rows ? a.g.gate_rows : a.g.T;
    const long slots_all = a.p.blocks * kSlots, first_group = a.p.own_groups ? blockIdx.x * kSlots + slot : blockIdx.x / a.p.per_group;
    const long r0 = first_group * G + (blockIdx.x % a.p.per_group) * a.p.rows_per_block;
    const long r1 = min(min(a.g.T, first_group * G + G), r0 + a.p.rows_per_block);
    const long turns = a.p.own_groups ? (a.p.groups + slots_all - 1) / slots_all * G : (a.p.rows_per_block + kSlots - 1) / kSlots;

    float w_post[CH][8], b_post[CH][8], w_pre[CH][8], gate[CH][8], total[kSums][CH][8];
#pragma unroll
    for (int c = 0; c < CH; ++c) {
        eight_weights(a.w.w_post, n[c], D, 1.f, w_post[c]);
        eight_weights(a.w.b_post, n[c], D, 0.f, b_post[c]);
        eight_weights(a.w.w_pre, n[c], D, 1.f, w_pre[c]);
#pragma unroll
        for (int k = 0; k < kSums; ++k)
#pragma unroll
            for (int e = 0; e < 8; ++e) total[k][c][e] = 0.f;
    }
    long group = -1, in_group = 0, own = first_group;
    for (long t = 0; t < turns; ++t) {
        long row = r0 + t * kSlots + slot;
        bool there = row < r1;
        long here = first_group;
        if (a.p.own_groups) {
            row = own * G + in_group;
            there = own < a.p.groups && row < a.g.T;
            here = own;
        }
        if (here != group && there) {
            group = here;
#pragma unroll
            for (int c = 0; c < CH; ++c) eight_weights(gated ? a.w.gate + here * D : nullptr, n[c], D, 1.f, gate[c]);
        }
        float f[CH][8], s[CH][8], g[CH][8], h[CH][8];
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            Eight<T> x[4];
            const float zero[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int k = 0; k < 4; ++k) x[k].set(zero);
            if (there && count[c]) {
                if (a.F) x[0] = read_eight((const T *)a.F + row * a.g.ld_f, n[c], D, a.wide_f);
                if (pre) x[1] = read_eight((const T *)a.S_in + row * D, n[c], D, a.wide);
                if (pre) x[2] = read_eight((const T *)a.dH + row * D, n[c], D, a.wide);
                if (a.dS) x[3] = read_eight((const T *)a.dS + row * D, n[c], D, a.wide);
            }
            x[0].get(f[c]);
            x[1].get(s[c]);
            x[2].get(h[c]);
            x[3].get(g[c]);
        }
        float2 of_s = make_float2(0.f, 1.f), of_f = make_float2(0.f, 1.f);
        if (post && pre) statistics2<WPR, CH>(a.g.pre, a.g.eps_pre, s, &of_s, a.g.post, a.g.eps_post, f, &of_f, count, a.inv_d, sum);
        else if (pre) of_s = statistics<WPR, CH>(a.g.pre, a.g.eps_pre, s, count, a.inv_d, sum);
        else if (post) of_f = statistics<WPR, CH>(a.g.post, a.g.eps_post, f, count, a.inv_d, sum);
        if (pre) {
            float mean = 0.f, along = 0.f;
#pragma unroll
            for (int c = 0; c < CH; ++c)
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    s[c][e] = (s[c][e] - of_s.x) * of_s.y;
                    if (there) total[kWPre][c][e] += h[c][e] * s[c][e];
                    total[kBPre][c][e] += h[c][e];
                    h[c][e] *= w_pre[c][e];
                    mean += h[c][e];
                    along += h[c][e] * s[c][e];
                }
            sum(mean, along);
            mean = a.g.pre == CAC_NORM_LAYER ? mean * a.inv_d : 0.f;
            along *= a.inv_d;
#pragma unroll
            for (int c = 0; c < CH; ++c)
#pragma unroll
                for (int e = 0; e < 8; ++e) g[c][e] += of_s.y * (h[c][e] - mean - s[c][e] * along);
        }
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            if (there && count[c] && a.dR) write_eight((T *)a.dR + row * D, n[c], D, a.wide, g[c]);
            drop_eight(key, a.d, (uint64_t)(row * across + (n[c] >> 3)), a.scale, g[c]);
#pragma unroll
            for (int e = 0; e < 8; ++e) g[c][e] = e < count[c] && there ? g[c][e] : 0.f;
        }
        if (there) {
#pragma unroll
            for (int c = 0; c < CH; ++c)
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    f[c][e] = (f[c][e] - of_f.x) * of_f.y;
                    total[kGate][c][e] += g[c][e] * (f[c][e] * w_post[c][e] + b_post[c][e]);
                    g[c][e] *= gate[c][e];
                    total[kWPost][c][e] += g[c][e] * f[c][e];
                    total[kBPost][c][e] += g[c][e];
                }
        }
        if (post) {
            float mean = 0.f, along = 0.f;
#pragma unroll
            for (int c = 0; c < CH; ++c)
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    g[c][e] *= w_post[c][e];
                    mean += g[c][e];
                    along += g[c][e] * f[c][e];
                }
            sum(mean, along);
            mean = a.g.post == CAC_NORM_LAYER ? mean * a.inv_d : 0.f;
            along *= a.inv_d;
#pragma unroll
            for (int c = 0; c < CH; ++c)
#pragma unroll
                for (int e = 0; e < 8; ++e) g[c][e] = of_f.y * (g[c][e] - mean - f[c][e] * along);
        }
#pragma unroll
        for (int c = 0; c < CH; ++c)
            if (there && count[c] && a.dF) write_eight((T *)a.dF + row * D, n[c], D, a.wide, g[c]);
        if (a.p.own_groups && (++in_group == G || t + 1 == turns)) { // a whole group's gate
            in_group = 0;
#pragma unroll
            for (int c = 0; c < CH; ++c) {
                if (own < a.p.groups && a.o.gate) write_eight(a.o.gate + own * D, n[c], D, D % 4 == 0 && n[c] + 8 <= D, total[kGate][c]);
#pragma unroll
                for (int e = 0; e < 8; ++e) total[kGate][c][e] = 0.f;
            }
            own += slots_all;
        }
    }

    float *const out[kSums] = {a.o.gate, a.o.w_post, a.o.b_post, a.o.w_pre, a.o.b_pre};
#pragma unroll
    for (int k = 0; k < kSums; ++k) {
        if (!out[k] || (k == kGate && a.p.own_groups)) continue;
        if (kSlots > 1) {
            const int at = (wave % WPR * 64 + lane) * 8; // (CH is 1 where there are slots)
            if (slot > 0) {
                Eight<float> x;
                x.set(total[k][0]);
                x.write(joined + (slot - 1) * kColumns + at);
            }
            __syncthreads();
            if (slot == 0)
                for (int i = 0; i < kSlots - 1; ++i)
#pragma unroll
                    for (int e = 0; e < 8; ++e) total[k][0][e] += joined[i * kColumns + at + e];
            __syncthreads();
        }
        if (slot > 0) continue;
        float *to = k == kGate ? (a.p.per_group == 1 ? out[k] + first_group * D : nullptr) : a.p.blocks == 1 ? out[k] : nullptr;
        if (!to) to = a.part + (k * a.p.blocks + blockIdx.x) * D;
#pragma unroll
        for (int c = 0; c < CH; ++c) write_eight(to, n[c], D, D % 4 == 0 && n[c] + 8 <= D, total[k][c]);
    }
}

// The workgroups' sums joined: a block of sixteen waves takes 64 columns of one vector.
__global__ void __launch_bounds__(1024) norm_join_kernel(const NormArgs a)
{
    __shared__ float red[16][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, D = (int)a.g.D, col = blockIdx.x * 64 + lane;
    const int k = blockIdx.y < 4 ? kWPost + blockIdx.y : kGate;
    const long group = blockIdx.y < 4 ? 0 : blockIdx.y - 4, rows = k == kGate ? a.p.per_group : a.p.blocks;
    float *to = k == kGate ? a.o.gate : k == kWPost ? a.o.w_post : k == kBPost ? a.o.b_post : k == kWPre ? a.o.w_pre : a.o.b_pre;
    if (!to) return;
    const float *p = a.part + (k * a.p.blocks + group * rows) * D + col;
    float s = 0.f;
    if (col < D) {
        long r = wave;
        for (; r + 48 < rows; r += 64) {
            const float x0 = p[r * D], x1 = p[(r + 16) * D], x2 = p[(r + 32) * D], x3 = p[(r + 48) * D];
            s += (x0 + x1) + (x2 + x3);
        }
        for (; r < rows; r += 16) s += p[r * D];
    }
    red[wave][lane] = s;
    __syncthreads();
    if (wave || col >= D) return;
    for (int w = 1; w < 16; ++w) s += red[w][lane];
    to[group * D + col] = s;
}

// ---- host
static long cdiv(long a, long b) { return (a + b - 1) / b; }

void plan_norm(const NormGeom &g, bool backward, NormPlan *p)
{
    p->chunks = g.D > 8192 ? 2 : 1;
    p->waves = 1;
    while (p->waves * 512 * p->chunks < g.D) p->waves *= 2;
    const int least = backward ? 8 : 4, waves = p->waves > least ? p->waves : least;
    p->slots = waves / p->waves;
    p->own_groups = false;
    p->groups = g.gate_rows ? cdiv(g.T, g.gate_rows) : 1;
    p->per_group = 1;
    if (!backward) {
        p->blocks = cdiv(g.T, p->slots);
        const long most = 256 * 16 / waves;
        if (p->blocks > most) p->blocks = most;
        p->rows_per_block = cdiv(g.T, p->blocks);
        p->blocks = cdiv(g.T, p->rows_per_block);
        p->bytes = 0;
        return;
    }
    const long most = 256 * 16 / waves, G = g.gate_rows ? g.gate_rows : g.T;
    if (p->groups > 1 && (p->groups * 2 >= most * p->slots || G <= 4)) {
        p->own_groups = true;
        p->blocks = cdiv(p->groups, p->slots);
        if (p->blocks > most) p->blocks = most;
        p->rows_per_block = 0;
    } else {
        const long per = most / p->groups > 0 ? most / p->groups : 1;
        p->rows_per_block = cdiv(G, per);
        if (p->rows_per_block < p->slots) p->rows_per_block = p->slots;
        p->per_group = cdiv(G, p->rows_per_block);
        p->blocks = p->groups * p->per_group;
    }
    p->bytes = p->blocks > 1 ? (size_t)kSums * p->blocks * g.D * sizeof(float) : 0;
}

static NormArgs arguments(const NormGeom &g, const NormPlan &p, const Drop &d, const NormParams &w)
{
    NormArgs a = {};
    a.g = g;
    a.p = p;
    a.d = d;
    a.w = w;
    a.scale = g.alpha * d.scale;
    a.inv_d = 1.f / (float)g.D;
    const long whole = g.dtype == CAC_F32 ? 4 : 8;
    a.wide = g.D % 8 == 0;
    a.wide_f = a.wide && g.ld_f % whole == 0;
    a.wide_r = a.wide && g.ld_r % whole == 0;
    return a;
}

template <typename T, int WPR, int CH> static hipError_t launch_of(const NormArgs &a, bool backward, hipStream_t st)
{
    if (backward) hipLaunchKernelGGL((norm_bwd_kernel<T, WPR, CH>), dim3((unsigned)a.p.blocks), dim3(64 * kBwdWaves<WPR>), 0, st, a);
    else hipLaunchKernelGGL((norm_fwd_kernel<T, WPR, CH>), dim3((unsigned)a.p.blocks), dim3(64 * kFwdWaves<WPR>), 0, st, a);
    return hipGetLastError();
}
template <typename T> static hipError_t launch_rows(const NormArgs &a, bool backward, hipStream_t st)
{
    if (a.p.chunks == 2) return launch_of<T, 16, 2>(a, backward, st);
    switch (a.p.waves) {
    case 1: return launch_of<T, 1, 1>(a, backward, st);
    case 2: return launch_of<T, 2, 1>(a, backward, st);
    case 4: return launch_of<T, 4, 1>(a, backward, st);
    case 8: return launch_of<T, 8, 1>(a, backward, st);
    default: return launch_of<T, 16, 1>(a, backward, st);
    }
}

hipError_t launch_norm_fwd(const NormGeom &g, const NormPlan &p, const Drop &d, const void *F, const void *R, const NormParams &w, void *S, void *H,
                           hipStream_t st)
{
    NormArgs a = arguments(g, p, d, w);
    a.F = F;
    a.R = R;
    a.S = S;
    a.H = H;
    return g.dtype == CAC_F32 ? launch_rows<float>(a, false, st) : launch_rows<bf16_t>(a, false, st);
}

hipError_t launch_norm_bwd(const NormGeom &g, const NormPlan &p, const Drop &d, const void *F, const void *S, const NormParams &w, const void *dH,
                           const void *dS, void *dR, void *dF, const NormGrads &o, void *ws, hipStream_t st)
{
    NormArgs a = arguments(g, p, d, w);
    a.F = F;
    a.S_in = S;
    a.dH = dH;
    a.dS = dS;
    a.dR = dR;
    a.dF = dF;
    a.o = o;
    a.part = (float *)ws;
    hipError_t e = g.dtype == CAC_F32 ? launch_rows<float>(a, true, st) : launch_rows<bf16_t>(a, true, st);
    if (e != hipSuccess || p.blocks == 1) return e;
    const bool gates = o.gate && !p.own_groups && p.per_group > 1;
    if (!gates && !o.w_post && !o.b_post && !o.w_pre && !o.b_pre) return hipSuccess;
    hipLaunchKernelGGL(norm_join_kernel, dim3((unsigned)cdiv(g.D, 64), (unsigned)(4 + (gates ? p.groups : 0))), dim3(1024), 0, st, a);
    return hipGetLastError();
}

} // namespace cac
