// What stands between two blocks of a residual network:
//   forward : S = R + alpha * drop(gate * post(F)),  H = pre(S)
//   backward: dR = dS + pre'(S)^T dH,  a = alpha * drop(dR),  dF = post'(F)^T (gate * a), and the sums over rows for the gate and the
//             norms' weights.
// A norm's statistics of a row are formed from the row in registers, in the forward pass and again in the backward pass, so that neither they
// nor the normalised row nor the mask is kept: what the backward pass reads is F and S.  With xhat = (x - mean) / sqrt(var + eps), g the gradient of
// xhat:  dx = (g - mean(g) - xhat mean(g xhat)) / sqrt(var + eps), without the first two means for rms.
// Bound by memory: every row is read and written once.  A row is spread over the lanes of a quarter of a wave to sixteen waves, eight
// neighbours to a lane (two groups of eight above 8192 columns); weights stay in registers while a workgroup goes from row to
// row, and so do the sums over rows, whose order is fixed: a workgroup's, then the workgroups'.
// Measured, bfloat16: forward 8192 x 4096 with both norms and dropout 56 us (4.8 TB/s; two streams in and two out copy at 5.15), vector instructions on
// 56 % of cycles; gradients 8192 x 2048 52 us, of which 13 are the first row's way, the ends and the joining of sums (8192 rows more take 39, 5.15 TB/s).
// One workgroup to a compute unit in the backward pass, since each leaves up to five vectors of partial sums: two take 66 us where one takes 60 (before other steps).
#include "block.h"

namespace cac {

struct NormArgs {
    int T, D, across;            // across: groups of eight to a row
    int post, pre;               // cac_norm
    int gate_rows, groups;       // rows that share a row of the gate (0: no gate), and how many such groups
    int rows_per_block, blocks, per_group;
    bool own;                    // backward: a slot has groups of the gate to itself
    long ld_f, ld_r;
    float eps_post, eps_pre;
    float scale;                 // alpha over the probability of being kept
    float inv_d;
    Drop d;
    NormParams w;
    const void *F, *R, *S_in, *dH, *dS;
    void *S, *H, *dR, *dF;
    NormGrads o;
    float *part;                 // [5][blocks][D], of the sums in NormGrads' order
    float *known;                // [T][8] of long rows: mean and inverse spread of F and of S, mean and projection of pre's gradient
};

// The sum over LANES neighbouring lanes in every one of them, in one order for all.
template <int LANES> __device__ __forceinline__ float lanes_total(float x)
{
    auto moved = [](float v, auto ctrl) { return __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(v), decltype(ctrl)::value, 0xf, 0xf, true)); };
    if (LANES >= 2) x += moved(x, std::integral_constant<int, 0xB1>());   // neighbours
    if (LANES >= 4) x += moved(x, std::integral_constant<int, 0x4E>());   // pairs
    if (LANES >= 8) x += moved(x, std::integral_constant<int, 0x141>());  // fours, mirrored
    if (LANES >= 16) x += moved(x, std::integral_constant<int, 0x140>()); // eights, mirrored
    if (LANES >= 32) {
        const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
        x = __uint_as_float(r[0]) + __uint_as_float(r[1]);
    }
    if (LANES >= 64) {
        const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
        x = __uint_as_float(r[0]) + __uint_as_float(r[1]);
    }
    return x;
}

// How a row lies in a workgroup: over LANES lanes of each of WPR waves, CH groups of eight to a lane.  WHOLE: rows are whole eights.
template <int LANES_, int WPR_, int CH_, bool WHOLE_> struct Rows {
    static constexpr int LANES = LANES_, WPR = WPR_, CH = CH_;
    static constexpr bool WHOLE = WHOLE_;
    static constexpr int kColumns = 8 * LANES * WPR * CH;
    static_assert(LANES == 64 || WPR == 1, "part of a wave, or waves");
    int n[CH], count[CH]; // the lane's first columns, and how many of its eights there are
    int from[CH];         // where its eights are read from: a row's end may lie inside
    int slot;             // which of the workgroup's rows
    __device__ __forceinline__ Rows(int D, int first = 0)
    {
        const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
        slot = LANES == 64 ? wave / WPR : (int)threadIdx.x / LANES;
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            n[c] = first + ((c * WPR + wave % WPR) * LANES + threadIdx.x % LANES) * 8;
            count[c] = min(max(D - n[c], 0), 8);
            from[c] = WHOLE ? n[c] : max(min(n[c], D - 8), 0);
        }
    }
    // Whole loads, a row's last eight where the lane's eights end past it; taken to their place when they have arrived, so that
    // nothing waits for them here.
    template <typename T> __device__ __forceinline__ Eight<T> ask(const T *row, int c, int D) const
    {
        if (!WHOLE && D < 8) return read_eight(row, n[c], D);
        Eight<T> r;
        r.read(row + from[c]);
        return r;
    }
    template <typename T> __device__ __forceinline__ void get(Eight<T> x, int c, float (&v)[8]) const
    {
        if (!WHOLE && n[c] != from[c]) x.shift(n[c] - from[c]);
        x.get(v);
    }
};

// Where the WPR waves of a row meet: lane i goes away with the numbers of wave i % kTurns, kTurns the power of two from WPR on, and with zeros where there is
// no such wave.  `red` holds two turns, so that one meeting is enough: a wave that writes a turn's numbers has met since the others read those of the turn
// before.
template <class L> struct Meeting {
    float *red; // [2][waves of the workgroup][8]
    int waves, turn;
    float columns; // of a row in the wave whose numbers the lane goes away with
    static constexpr int kTurns = L::WPR <= 1 ? 1 : L::WPR <= 2 ? 2 : L::WPR <= 4 ? 4 : L::WPR <= 8 ? 8 : 16;
    __device__ __forceinline__ Meeting(float *lds, int all, int D) : red(lds), waves(all), turn(0)
    {
        const int w = (threadIdx.x & 63) % kTurns;
        int n = 0;
#pragma unroll
        for (int c = 0; c < L::CH; ++c)
            if (w < L::WPR) n += min(max(D - (c * L::WPR + w) * L::LANES * 8, 0), L::LANES * 8);
        columns = (float)n;
    }
    // of which a wave's lanes all have the same
    template <int N> __device__ __forceinline__ void operator()(float (&x)[N])
    {
        static_assert(N <= 8, "eight to a wave");
        if (L::WPR == 1) return;
        float *r = red + turn * waves * 8;
        const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
        if (lane == 0) {
#pragma unroll
            for (int i = 0; i < N; ++i) r[wave * 8 + i] = x[i];
        }
        __syncthreads();
        const int w = lane % kTurns;
        r += (wave / L::WPR * L::WPR + min(w, L::WPR - 1)) * 8;
#pragma unroll
        for (int i = 0; i < N; ++i) x[i] = w < L::WPR ? r[i] : 0.f;
        turn ^= 1;
    }
    // over a row's waves, of a number that lane i has of wave i % kTurns
    __device__ __forceinline__ float total(float x) const { return lanes_total<kTurns>(x); }
};

// 1 / sqrt(x): the instruction's 22 bits, and a step of Newton's.  The instruction takes numbers below the least normal one for zeros, so small ones go
// through it times 2^64.
__device__ __forceinline__ float inverse_root(float x)
{
    const bool small = x < 0x1p-100f;
    const float z = small ? x * 0x1p64f : x, y = __builtin_amdgcn_rsqf(z), r = fmaf(-z * y, y, 1.f);
    return (x > 0.f && x < INFINITY ? fmaf(0.5f * y, r, y) : y) * (small ? 0x1p32f : 1.f);
}

// eight of a vector of weights, `otherwise` where there is none, zeros past its end
__device__ __forceinline__ void eight_weights(const float *w, int n, int count, float otherwise, float (&v)[8])
{
    if (w && count == 8) {
        Eight<float> x;
        x.read(w + n);
        x.get(v);
        return;
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = e < count ? (w ? w[n + e] : otherwise) : 0.f;
}

// Sum of a row's (x - mean)^2 in a lane.  What is read past a row's end is zero, and the mean away from it.
template <class L> __device__ __forceinline__ float squares(int kind, const float (&x)[L::CH][8], float mean, const L &l)
{
    float v = 0.f;
#pragma unroll
    for (int c = 0; c < L::CH; ++c) {
        float u = 0.f;
        if (kind == CAC_NORM_RMS) {
#pragma unroll
            for (int e = 0; e < 8; ++e) u += x[c][e] * x[c][e];
        } else if (L::WHOLE) {
#pragma unroll
            for (int e = 0; e < 8; ++e) u += (x[c][e] - mean) * (x[c][e] - mean);
            u = l.count[c] ? u : 0.f;
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float y = e < l.count[c] ? x[c][e] - mean : 0.f;
                u += y * y;
            }
        }
        v += u;
    }
    return v;
}
template <class L> __device__ __forceinline__ float lane_sum(const float (&x)[L::CH][8])
{
    float v = 0.f;
#pragma unroll
    for (int c = 0; c < L::CH; ++c)
#pragma unroll
        for (int e = 0; e < 8; ++e) v += x[c][e];
    return v;
}

// A row's mean and the sum of squares about it come from one meeting: each wave has its own mean and the squares about that, and
//   sum (x - mean)^2 = sum over waves of (squares about the wave's mean + columns (wave's mean - mean)^2).
struct Stats { float mean, inv; }; // mean is 0 for rms
template <class L> __device__ __forceinline__ float wave_mean(int kind, const float (&x)[L::CH][8], const Meeting<L> &meet)
{
    if (kind != CAC_NORM_LAYER) return 0.f;
    const float n = L::WPR == 1 ? meet.columns : __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(meet.columns), __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) % L::WPR));
    return lanes_total<L::LANES>(lane_sum<L>(x)) * __builtin_amdgcn_rcpf(fmaxf(n, 1.f)); // (any number near the mean will do, the same for all)
}
// from the waves' means m and squares q
template <class L> __device__ __forceinline__ Stats joined_stats(int kind, float eps, float m, float q, float inv_d, const Meeting<L> &meet)
{
    float mean = 0.f;
    if (kind == CAC_NORM_LAYER && L::WPR == 1) mean = m;
    if (kind == CAC_NORM_LAYER && L::WPR > 1) {
        mean = meet.total(meet.columns * m) * inv_d;
        q += meet.columns * ((m - mean) * (m - mean));
    }
    return Stats{mean, inverse_root(meet.total(q) * inv_d + eps)};
}
template <class L> __device__ __forceinline__ Stats statistics(int kind, float eps, const float (&x)[L::CH][8], const L &l, const NormArgs &a, Meeting<L> &meet)
{
    float of[2];
    of[0] = wave_mean<L>(kind, x, meet);
    of[1] = lanes_total<L::LANES>(squares(kind, x, of[0], l));
    meet(of);
    return joined_stats<L>(kind, eps, of[0], of[1], a.inv_d, meet);
}
// the row before weights
template <class L> __device__ __forceinline__ void normalise(int kind, Stats s, float (&x)[L::CH][8])
{
    if (kind == CAC_NORM_NONE) return;
    if (kind == CAC_NORM_LAYER) {
#pragma unroll
        for (int c = 0; c < L::CH; ++c)
#pragma unroll
            for (int e = 0; e < 8; ++e) x[c][e] -= s.mean;
    }
#pragma unroll
    for (int c = 0; c < L::CH; ++c)
#pragma unroll
        for (int e = 0; e < 8; ++e) x[c][e] *= s.inv;
}
// g, the gradient of the normalised row x, to that of the row, which is added to `to`; mean: of g (0 for rms), along: of g x
template <class L> __device__ __forceinline__ void add_gradient(float inv, float mean, float along, const float (&x)[L::CH][8], const float (&g)[L::CH][8], float (&to)[L::CH][8])
{
#pragma unroll
    for (int c = 0; c < L::CH; ++c)
#pragma unroll
        for (int e = 0; e < 8; ++e) to[c][e] += inv * (g[c][e] - mean - x[c][e] * along);
}

template <int WPR> constexpr int kFwdWaves = WPR > 4 ? WPR : 4;
template <int WPR> constexpr int kBwdWaves = WPR > 8 ? WPR : 8;

template <typename T, class L> __global__ void __launch_bounds__(64 * kFwdWaves<L::WPR>) norm_fwd_kernel(const NormArgs a)
{
    constexpr int kWaves = kFwdWaves<L::WPR>, kSlots = kWaves * 64 / L::LANES / L::WPR, CH = L::CH;
    __shared__ float red[16 * kWaves];
    const int D = a.D;
    const L l(D);
    Meeting<L> meet(red, kWaves, D);
    const int r0 = blockIdx.x * a.rows_per_block, r1 = min(a.T, r0 + a.rows_per_block);
    const DropKey key = drop_key(a.d);
    Eight<T> f[CH], r[CH];
    auto ask = [&](long row) {
#pragma unroll
        for (int c = 0; c < CH; ++c)
            if (l.count[c]) {
                f[c] = l.ask((const T *)a.F + row * a.ld_f, c, D);
                if (a.R) r[c] = l.ask((const T *)a.R + row * a.ld_r, c, D);
            }
    };
#pragma unroll
    for (int c = 0; c < CH; ++c) {
        f[c].clear();
        r[c].clear();
    }
    if (r0 + l.slot < r1) ask(r0 + l.slot);
    // post's weights, the gate and the branch's factor as one factor and one summand, zeros past a row's end
    float w_pre[CH][8], b_pre[CH][8], factor[CH][8], summand[CH][8];
#pragma unroll
    for (int c = 0; c < CH; ++c) {
        eight_weights(a.w.w_pre, l.n[c], l.count[c], 1.f, w_pre[c]);
        eight_weights(a.w.b_pre, l.n[c], l.count[c], 0.f, b_pre[c]);
    }
    int group = -1, last = -1; // the gate's row at hand, and the last of T that it is of
    for (int base = r0; base < r1; base += kSlots) {
        const int row = base + l.slot;
        const bool there = row < r1;
        float v[CH][8], s[CH][8];
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            l.get(f[c], c, v[c]);
            l.get(r[c], c, s[c]);
        }
        if (row + kSlots < r1) ask(row + kSlots);
        if (row > last) {
            group = a.gate_rows && there ? row / a.gate_rows : 0;
            last = a.gate_rows && there ? group * a.gate_rows + a.gate_rows - 1 : a.T;
#pragma unroll
            for (int c = 0; c < CH; ++c) {
                float gate[8];
                eight_weights(a.w.w_post, l.n[c], l.count[c], 1.f, factor[c]);
                eight_weights(a.w.b_post, l.n[c], l.count[c], 0.f, summand[c]);
                eight_weights(a.w.gate ? a.w.gate + (long)group * D : nullptr, l.n[c], l.count[c], 1.f, gate);
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    factor[c][e] *= gate[e] * a.scale;
                    summand[c][e] *= gate[e] * a.scale;
                }
            }
        }
        if (a.post != CAC_NORM_NONE) normalise<L>(a.post, statistics(a.post, a.eps_post, v, l, a, meet), v);
#pragma unroll
        for (int c = 0; c < CH; ++c) {
#pragma unroll
            for (int e = 0; e < 8; ++e) v[c][e] = v[c][e] * factor[c][e] + summand[c][e];
            drop_eight(key, a.d, (uint64_t)row * a.across + (l.n[c] >> 3), v[c]);
#pragma unroll
            for (int e = 0; e < 8; ++e) s[c][e] += v[c][e];
            if (there && l.count[c] && a.S) write_eight<L::WHOLE>((T *)a.S + (long)row * D, l.n[c], D, s[c]);
        }
        if (!a.H) continue;
        normalise<L>(a.pre, statistics(a.pre, a.eps_pre, s, l, a, meet), s);
#pragma unroll
        for (int c = 0; c < CH; ++c) {
#pragma unroll
            for (int e = 0; e < 8; ++e) s[c][e] = s[c][e] * w_pre[c][e] + b_pre[c][e];
            if (there && l.count[c]) write_eight<L::WHOLE>((T *)a.H + (long)row * D, l.n[c], D, s[c]);
        }
    }
}

enum { kGate, kWPost, kBPost, kWPre, kBPre, kSums };

// The sums over rows that the gate and post's weights need are two, of a and of a xhat, as long as the gate is the same:
//   dgate = w sum(a xhat) + b sum(a),  dw = gate sum(a xhat),  db = gate sum(a).
// A workgroup has rows of one group (a run of them, its slots taking turns); or (own_groups) every slot has groups to itself, and adds
// a group's sums up in LDS when it ends.
// Both parts in one pass where a workgroup's registers hold a row and its sums; of longer rows the row part leaves what it knows of a row, eight numbers,
// and the sum part has 512 columns to a workgroup and reads the rows again.
enum Part { kBoth, kRowPart, kSumPart };
template <typename T, class L, Part PART> __global__ void __launch_bounds__(64 * kBwdWaves<L::WPR>, kBwdWaves<L::WPR> / 4) norm_bwd_kernel(const NormArgs a)
{
    constexpr int kWaves = kBwdWaves<L::WPR>, kThreads = 64 * kWaves, kSlots = kThreads / L::LANES / L::WPR, CH = L::CH;
    constexpr bool kTakesSums = PART != kRowPart, kAhead = L::WPR < 16; // (else there are no registers for a row ahead, and a row is enough on its way)
    __shared__ float red[16 * kWaves];
    __shared__ float kept[kTakesSums ? 2 : 1][CH][8][kTakesSums ? kThreads : 1]; // own_groups: sums for w_post and b_post
    __shared__ float joined[kSlots > 1 ? kThreads * 8 : 1];
    const int D = a.D;
    const L l(D, PART == kSumPart ? blockIdx.y * L::kColumns : 0);
    Meeting<L> meet(red, kWaves, D);
    const DropKey key = drop_key(a.d);
    const bool post = a.post != CAC_NORM_NONE, pre = a.pre != CAC_NORM_NONE, own = a.own, wants_a = a.o.b_post || (a.o.gate && a.w.b_post);

    const int rows = a.T, G = a.gate_rows ? a.gate_rows : rows, slots_all = a.blocks * kSlots, groups = a.groups;
    int group = own ? blockIdx.x * kSlots + l.slot : blockIdx.x / (unsigned)a.per_group;
    const int per_block = a.rows_per_block, r0 = group * (own ? 0 : G) + blockIdx.x % (unsigned)a.per_group * per_block;
    const int r1 = min(rows, min(own ? 0 : group * G + G, r0 + per_block));
    const int turns = own ? (groups + slots_all - 1) / slots_all * G : (per_block + kSlots - 1) / kSlots;
    // the row of a turn, or one past the last
    int asked = r0 + l.slot, asked_group = group;
    if (own) asked = 0;
    auto next_row = [&]() {
        int row = asked;
        if (!own) {
            asked += kSlots;
            return row < r1 ? row : rows;
        }
        row = asked_group < groups ? min(asked_group * G + row, rows) : rows;
        if (++asked == G) {
            asked = 0;
            asked_group += slots_all;
        }
        return row;
    };
    Eight<T> x[4][CH];
    auto ask = [&](long row) {
        if (row >= rows) return;
#pragma unroll
        for (int c = 0; c < CH; ++c)
            if (l.count[c]) {
                if (a.F) x[0][c] = l.ask((const T *)a.F + row * a.ld_f, c, D);
                if (pre) x[1][c] = l.ask((const T *)a.S_in + row * D, c, D);
                if (pre) x[2][c] = l.ask((const T *)a.dH + row * D, c, D);
                if (a.dS) x[3][c] = l.ask((const T *)a.dS + row * D, c, D);
            }
    };
#pragma unroll
    for (int k = 0; k < 4; ++k)
#pragma unroll
        for (int c = 0; c < CH; ++c) x[k][c].clear();

    int now = kAhead ? next_row() : 0, in_group = 0;
    if (kAhead) ask(now); // (before the weights, whose products are waited for)
    float w_pre[CH][8], factor[CH][8], sum_a[CH][8], sum_ax[CH][8], sum_h[CH][8], sum_hx[CH][8];
    auto gate_factor = [&](int g) { // gate times w_post times the branch's factor, zeros past a row's end
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            float gate[8];
            eight_weights(a.w.w_post, l.n[c], l.count[c], 1.f, factor[c]);
            eight_weights(a.w.gate && g < groups ? a.w.gate + (long)g * D : nullptr, l.n[c], l.count[c], 1.f, gate);
#pragma unroll
            for (int e = 0; e < 8; ++e) factor[c][e] *= gate[e] * a.scale;
        }
    };
#pragma unroll
    for (int c = 0; c < CH; ++c) {
        eight_weights(a.w.w_pre, l.n[c], l.count[c], 1.f, w_pre[c]);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            sum_a[c][e] = sum_ax[c][e] = sum_h[c][e] = sum_hx[c][e] = 0.f;
            if constexpr (kTakesSums)
                if (own) kept[0][c][e][threadIdx.x] = kept[1][c][e][threadIdx.x] = 0.f;
        }
    }
    gate_factor(group);
    for (int t = 0; t < turns; ++t) {
        if (!kAhead) ask(now = next_row());
        const long row = now;
        const bool there = now < rows;
        if (kAhead) now = t + 1 < turns ? next_row() : rows;
        float f[CH][8], s[CH][8], g[CH][8], h[CH][8];
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            l.get(x[0][c], c, f[c]);
            l.get(x[1][c], c, s[c]);
            l.get(x[2][c], c, h[c]);
            l.get(x[3][c], c, g[c]);
        }
        if (kAhead) ask(now);
        Stats of_s = {0.f, 1.f}, of_f = {0.f, 1.f};
        float mean = 0.f, along = 0.f; // of pre's gradient
        if constexpr (PART == kSumPart) {
            const float *k = a.known + (there ? row : 0) * 8;
            of_f = Stats{k[0], k[1]};
            of_s = Stats{k[2], k[3]};
            mean = k[4];
            along = k[5];
        } else {
            float first[6] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f}; // means and squares of F and S; sums of w dH and w dH (S - S's mean)
            if (post) {
                first[0] = wave_mean<L>(a.post, f, meet);
                first[1] = lanes_total<L::LANES>(squares(a.post, f, first[0], l));
            }
            if (pre) {
                first[2] = wave_mean<L>(a.pre, s, meet);
                first[3] = lanes_total<L::LANES>(squares(a.pre, s, first[2], l));
                float with = 0.f;
#pragma unroll
                for (int c = 0; c < CH; ++c)
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        const float hw = h[c][e] * w_pre[c][e];
                        first[4] += hw;
                        with += hw * (s[c][e] - first[2]);
                    }
                if (a.pre == CAC_NORM_LAYER) first[4] = lanes_total<L::LANES>(first[4]);
                first[5] = lanes_total<L::LANES>(with);
            }
            if (post || pre) meet(first);
            if (post) of_f = joined_stats<L>(a.post, a.eps_post, first[0], first[1], a.inv_d, meet);
            if (pre) {
                of_s = joined_stats<L>(a.pre, a.eps_pre, first[2], first[3], a.inv_d, meet);
                along = first[5];
                if (a.pre == CAC_NORM_LAYER) {
                    mean = meet.total(first[4]) * a.inv_d;
                    if (L::WPR > 1) along += (first[2] - of_s.mean) * first[4];
                }
                along = meet.total(along) * (of_s.inv * a.inv_d);
            }
            if (PART == kRowPart && there && threadIdx.x == 0) {
                float *k = a.known + row * 8;
                k[0] = of_f.mean, k[1] = of_f.inv, k[2] = of_s.mean, k[3] = of_s.inv, k[4] = mean, k[5] = along;
            }
        }
        if (pre) {
            normalise<L>(a.pre, of_s, s);
            if (kTakesSums && there) {
#pragma unroll
                for (int c = 0; c < CH; ++c)
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        sum_hx[c][e] += h[c][e] * s[c][e];
                        sum_h[c][e] += h[c][e];
                    }
            }
#pragma unroll
            for (int c = 0; c < CH; ++c)
#pragma unroll
                for (int e = 0; e < 8; ++e) h[c][e] *= w_pre[c][e];
            add_gradient<L>(of_s.inv, mean, along, s, h, g);
        }
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            if (PART != kSumPart && there && l.count[c] && a.dR) write_eight<L::WHOLE>((T *)a.dR + row * D, l.n[c], D, g[c]);
            drop_eight(key, a.d, (uint64_t)row * a.across + (l.n[c] >> 3), g[c]); // (the factor comes last, to these and to the sums of them)
        }
        if (post) normalise<L>(a.post, of_f, f);
        if (kTakesSums && there) {
#pragma unroll
            for (int c = 0; c < CH; ++c)
#pragma unroll
                for (int e = 0; e < 8; ++e) sum_ax[c][e] += g[c][e] * f[c][e];
            if (wants_a) {
#pragma unroll
                for (int c = 0; c < CH; ++c)
#pragma unroll
                    for (int e = 0; e < 8; ++e) sum_a[c][e] += g[c][e];
            }
        }
        if constexpr (PART != kSumPart) {
#pragma unroll
            for (int c = 0; c < CH; ++c)
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    g[c][e] *= factor[c][e];
                    h[c][e] = 0.f;
                }
            if (post) {
                float second[2] = {0.f, 0.f};
#pragma unroll
                for (int c = 0; c < CH; ++c)
#pragma unroll
                    for (int e = 0; e < 8; ++e) second[1] += g[c][e] * f[c][e];
                if (a.post == CAC_NORM_LAYER) second[0] = lanes_total<L::LANES>(lane_sum<L>(g));
                second[1] = lanes_total<L::LANES>(second[1]);
                meet(second);
                add_gradient<L>(of_f.inv, a.post == CAC_NORM_LAYER ? meet.total(second[0]) * a.inv_d : 0.f, meet.total(second[1]) * a.inv_d, f, g, h);
            }
#pragma unroll
            for (int c = 0; c < CH; ++c)
                if (there && l.count[c] && a.dF) write_eight<L::WHOLE>((T *)a.dF + row * D, l.n[c], D, post ? h[c] : g[c]);
        }
        if (own && ++in_group == G) { // a whole group's
            in_group = 0;
            if constexpr (kTakesSums)
                if (group < groups)
#pragma unroll
                    for (int c = 0; c < CH; ++c) {
                        float w[8], b[8];
                        eight_weights(a.w.gate + (long)group * D, l.n[c], l.count[c], 1.f, w);
#pragma unroll
                        for (int e = 0; e < 8; ++e) {
                            kept[0][c][e][threadIdx.x] += w[e] * (a.scale * sum_ax[c][e]);
                            kept[1][c][e][threadIdx.x] += w[e] * (a.scale * sum_a[c][e]);
                        }
                        eight_weights(a.w.w_post, l.n[c], l.count[c], 1.f, w);
                        eight_weights(a.w.b_post, l.n[c], l.count[c], 0.f, b);
#pragma unroll
                        for (int e = 0; e < 8; ++e) {
                            w[e] = a.scale * (w[e] * sum_ax[c][e] + b[e] * sum_a[c][e]);
                            sum_ax[c][e] = sum_a[c][e] = 0.f;
                        }
                        if (a.o.gate && l.count[c]) write_eight(a.o.gate + (long)group * D, l.n[c], D, w);
                    }
            group += slots_all;
            gate_factor(group);
        }
    }

    if constexpr (!kTakesSums) return;
    float *const out[kSums] = {a.o.gate, a.o.w_post, a.o.b_post, a.o.w_pre, a.o.b_pre};
#pragma unroll
    for (int k = 0; k < kSums; ++k) {
        if (!out[k] || (k == kGate && own)) continue;
        float *to = k == kGate ? (a.per_group == 1 ? out[k] + (long)group * D : nullptr) : a.blocks == 1 ? out[k] : nullptr;
        if (!to) to = a.part + ((long)k * a.blocks + blockIdx.x) * D;
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            float v[8];
            if (k == kWPre || k == kBPre) {
#pragma unroll
                for (int e = 0; e < 8; ++e) v[e] = k == kWPre ? sum_hx[c][e] : sum_h[c][e];
            } else if (own) {
#pragma unroll
                for (int e = 0; e < 8; ++e) v[e] = kept[kTakesSums && k != kWPost ? 1 : 0][c][e][kTakesSums ? threadIdx.x : 0];
            } else {
                float w[8], b[8];
                eight_weights(k == kGate ? a.w.w_post : a.w.gate ? a.w.gate + (long)group * D : nullptr, l.n[c], l.count[c], 1.f, w);
                eight_weights(a.w.b_post, l.n[c], l.count[c], 0.f, b);
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    v[e] = a.scale * (k == kGate ? w[e] * sum_ax[c][e] + b[e] * sum_a[c][e] : w[e] * (k == kWPost ? sum_ax[c][e] : sum_a[c][e]));
            }
            if (kSlots > 1) { // (CH is 1 where there are slots)
                Eight<float> y;
                y.set(v);
                y.write(joined + l.slot * L::kColumns + l.n[0] % L::kColumns);
                __syncthreads();
                if (l.slot == 0)
                    for (int i = 1; i < kSlots; ++i) {
                        float u[8];
                        y.read(joined + i * L::kColumns + l.n[0] % L::kColumns);
                        y.get(u);
#pragma unroll
                        for (int e = 0; e < 8; ++e) v[e] += u[e];
                    }
                __syncthreads();
            }
            if (l.slot == 0 && l.count[c]) write_eight(to, l.n[c], D, v);
        }
    }
}

// The workgroups' sums joined: a block of sixteen waves takes 64 columns of one vector.
__global__ void __launch_bounds__(1024) norm_join_kernel(const NormArgs a)
{
    __shared__ float red[16][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, D = a.D, col = blockIdx.x * 64 + lane;
    const int k = blockIdx.y < 4 ? kWPost + blockIdx.y : kGate;
    const long group = blockIdx.y < 4 ? 0 : blockIdx.y - 4, rows = k == kGate ? a.per_group : a.blocks;
    float *to = k == kGate ? a.o.gate : k == kWPost ? a.o.w_post : k == kBPost ? a.o.b_post : k == kWPre ? a.o.w_pre : a.o.b_pre;
    if (!to) return;
    const float *p = a.part + ((long)k * a.blocks + group * rows) * D + col;
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

// Which rows a workgroup of the backward pass has, of `slots` at once and `most` workgroups at a time.  Where gates are many a slot has whole groups to
// itself, or a workgroup has (part of) one group: whichever takes fewer turns of a slot, 2 to 3 us each, where every round of workgroups costs as much as 4 turns
// more and one for sixteen slots whose sums it joins.  Gradients of bfloat16 with both norms, us, slots with groups of their own / workgroups with one:
//   2048 columns, gates of 49 rows: 255 gates 122 / 74, 256 gates 122 / 76, 257 122 / 130, 512 134 / 142, 513 229 / 195, 1024 254 / 276
//   4608 x 196: 127 gates 572 / 333, 128 572 / 337, 129 572 / 568.  1024 x 16: 511 46 / 38, 512 46 / 38, 513 46 / 48, 1024 49 / 70
//   128 x 49: 1024 gates 97 / 65, 2048 97 / 123, 4096 115 / 249.  2048 x 3: 128 17 / 22, 256 18 / 18, 512 21 / 29
static NormSplit split_rows(const NormGeom &g, long groups, int slots, long most)
{
    NormSplit s;
    const long G = g.gate_rows ? g.gate_rows : g.T;
    const long per = most / groups > 0 ? most / groups : 1;
    s.rows_per_block = cdiv(G, per);
    if (s.rows_per_block < slots) s.rows_per_block = slots;
    s.per_group = cdiv(G, s.rows_per_block);
    s.blocks = groups * s.per_group;
    const double round = 4.0 + slots / 16.0;
    const double turns = cdiv(s.blocks, most) * (cdiv(s.rows_per_block, slots) + round), turns_own = (double)cdiv(groups, most * slots) * G + round;
    s.own_groups = groups > 1 && turns_own <= turns;
    if (s.own_groups) {
        s.per_group = 1;
        s.rows_per_block = 0;
        s.blocks = cdiv(groups, slots);
        if (s.blocks > most) s.blocks = most;
    }
    return s;
}

void plan_norm(const NormGeom &g, bool backward, NormPlan *p)
{
    *p = NormPlan{};
    p->lanes = g.D <= 128 ? 16 : g.D <= 256 ? 32 : 64;
    p->chunks = g.D > 8192 ? 2 : 1;
    p->waves = 1;
    while (p->waves * 512 * p->chunks < g.D) p->waves *= 2;
    // Gradients of rows that twelve waves hold are faster with them than with sixteen, of which each then has registers for a row ahead (7523 x 4428 floats
    // 177 us against 332, 4000 x 6144 bf16 73 against 132 and floats 144 against 162); outputs are slower (4000 x 6144 bf16 64 against 51).
    if (backward && p->waves == 16 && g.D <= 12 * 512) p->waves = 12;
    const int least = backward ? 8 : 4, waves = p->waves > least ? p->waves : least;
    p->slots = waves * 64 / p->lanes / p->waves;
    p->groups = g.gate_rows ? cdiv(g.T, g.gate_rows) : 1;
    if (!backward) {
        const long most = 256 * 16 / waves; // (all at once)
        p->split.blocks = cdiv(g.T, p->slots);
        if (p->split.blocks > most) p->split.blocks = most;
        p->split.rows_per_block = cdiv(g.T, p->split.blocks);
        p->split.blocks = cdiv(g.T, p->split.rows_per_block);
        return;
    }
    p->split = split_rows(g, p->groups, p->slots, 256);
    p->two = g.D > 8192;
    p->sums = p->two ? split_rows(g, p->groups, 8, cdiv(1024, cdiv(g.D, 512))) : p->split;
    p->bytes = p->sums.blocks > 1 ? (size_t)kSums * p->sums.blocks * g.D * sizeof(float) : 0;
    p->bytes = (p->bytes + 255) / 256 * 256;
    p->o_known = p->bytes;
    if (p->two) p->bytes += (size_t)g.T * 8 * sizeof(float);
}

static void use(NormArgs &a, const NormSplit &s)
{
    a.rows_per_block = (int)s.rows_per_block;
    a.blocks = (int)s.blocks;
    a.per_group = (int)s.per_group;
    a.own = s.own_groups;
}

static NormArgs arguments(const NormGeom &g, const NormPlan &p, const Drop &d, const NormParams &w)
{
    NormArgs a = {};
    a.T = (int)g.T;
    a.D = (int)g.D;
    a.across = (int)cdiv(g.D, 8);
    a.post = g.post;
    a.pre = g.pre;
    a.gate_rows = (int)g.gate_rows;
    a.groups = (int)p.groups;
    use(a, p.split);
    a.ld_f = g.ld_f;
    a.ld_r = g.ld_r;
    a.eps_post = g.eps_post;
    a.eps_pre = g.eps_pre;
    a.scale = g.alpha * d.scale;
    a.inv_d = 1.f / (float)g.D;
    a.d = d;
    a.w = w;
    return a;
}

template <typename T, class L> static hipError_t launch_fwd(const NormArgs &a, hipStream_t st)
{
    hipLaunchKernelGGL((norm_fwd_kernel<T, L>), dim3((unsigned)a.blocks), dim3(64 * kFwdWaves<L::WPR>), 0, st, a);
    return hipGetLastError();
}
template <typename T, class L, Part PART = kBoth> static hipError_t launch_bwd(const NormArgs &a, hipStream_t st)
{
    const unsigned across = PART == kSumPart ? (unsigned)cdiv(a.D, L::kColumns) : 1;
    hipLaunchKernelGGL((norm_bwd_kernel<T, L, PART>), dim3((unsigned)a.blocks, across), dim3(64 * kBwdWaves<L::WPR>), 0, st, a);
    return hipGetLastError();
}
template <typename T, bool WHOLE> static hipError_t launch_rows(NormArgs a, const NormPlan &p, bool backward, hipStream_t st)
{
#define CAC_ROWS(LANES, WPR) \
    return backward ? launch_bwd<T, Rows<LANES, WPR, 1, WHOLE>>(a, st) : launch_fwd<T, Rows<LANES, WPR, 1, WHOLE>>(a, st)
    if (p.two) {
        hipError_t e = launch_bwd<T, Rows<64, 16, 2, WHOLE>, kRowPart>(a, st);
        if (e != hipSuccess || !(a.o.gate || a.o.w_post || a.o.b_post || a.o.w_pre || a.o.b_pre)) return e;
        use(a, p.sums);
        return launch_bwd<T, Rows<64, 1, 1, WHOLE>, kSumPart>(a, st);
    }
    if (p.chunks == 2) return launch_fwd<T, Rows<64, 16, 2, WHOLE>>(a, st);
    if (p.lanes == 16) CAC_ROWS(16, 1);
    if (p.lanes == 32) CAC_ROWS(32, 1);
    switch (p.waves) {
    case 1: CAC_ROWS(64, 1);
    case 2: CAC_ROWS(64, 2);
    case 4: CAC_ROWS(64, 4);
    case 8: CAC_ROWS(64, 8);
    case 12: return launch_bwd<T, Rows<64, 12, 1, WHOLE>>(a, st); // only gradients have them
    default: CAC_ROWS(64, 16);
    }
#undef CAC_ROWS
}
static hipError_t launch_norm(const NormArgs &a, const NormPlan &p, int dtype, bool backward, hipStream_t st)
{
    if (dtype == CAC_F32) return a.D % 8 ? launch_rows<float, false>(a, p, backward, st) : launch_rows<float, true>(a, p, backward, st);
    return a.D % 8 ? launch_rows<bf16_t, false>(a, p, backward, st) : launch_rows<bf16_t, true>(a, p, backward, st);
}

hipError_t launch_norm_fwd(const NormGeom &g, const NormPlan &p, const Drop &d, const void *F, const void *R, const NormParams &w, void *S, void *H,
                           hipStream_t st)
{
    NormArgs a = arguments(g, p, d, w);
    a.F = F;
    a.R = R;
    a.S = S;
    a.H = H;
    return launch_norm(a, p, g.dtype, false, st);
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
    a.known = (float *)((char *)ws + p.o_known);
    hipError_t e = launch_norm(a, p, g.dtype, true, st);
    if (e != hipSuccess || p.sums.blocks == 1) return e;
    const bool gates = o.gate && !p.sums.own_groups && p.sums.per_group > 1;
    if (!gates && !o.w_post && !o.b_post && !o.w_pre && !o.b_pre) return hipSuccess;
    use(a, p.sums);
    hipLaunchKernelGGL(norm_join_kernel, dim3((unsigned)cdiv(g.D, 64), (unsigned)(4 + (gates ? p.groups : 0))), dim3(1024), 0, st, a);
    return hipGetLastError();
}

} // namespace cac
