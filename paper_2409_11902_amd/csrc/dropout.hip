// Dropout with its residual, Y = R + alpha * drop(X): a thread has groups of eight neighbours of a row, whose random bits it forms once.
// Bound by memory (dropout.h): X and R in and Y out, once; 16384 x 4096 bfloat16 with R in 72 us, 5.57 TB/s.
#include "block.h"

namespace cac {

constexpr int kThreads = 256;

struct DropArgs {
    long groups;       // of all rows
    int wide;          // of a row
    long step_rows;    // what a thread's next group is away: rows and groups of a row
    int step_cols;
    int cols;
    long ld_x, ld_r;
    float scale;
    Drop d;
};

template <typename T, bool RES, bool WHOLE> __global__ void __launch_bounds__(kThreads) dropout_kernel(const DropArgs a, const T *X, const T *R, T *Y)
{
    const DropKey key = drop_key(a.d);
    const long stride = (long)gridDim.x * kThreads;
    long g = (long)blockIdx.x * kThreads + threadIdx.x;
    long row = a.groups >> 32 ? g / a.wide : (long)((uint32_t)g / (uint32_t)a.wide);
    int col = (int)(g - row * a.wide);
    for (; g < a.groups; g += stride) {
        const int n = col * 8;
        Eight<T> x = read_eight<WHOLE>(X + row * a.ld_x, n, a.cols), r;
        if (RES) r = read_eight<WHOLE>(R + row * a.ld_r, n, a.cols);
        float v[8];
        x.get(v);
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] *= a.scale;
        drop_eight(key, a.d, (uint64_t)g, v);
        if (RES) {
            float w[8];
            r.get(w);
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] += w[e];
        }
        write_eight<WHOLE>(Y + row * a.cols, n, a.cols, v);
        row += a.step_rows;
        col += a.step_cols;
        if (col >= a.wide) {
            col -= a.wide;
            ++row;
        }
    }
}

template <typename T> static hipError_t launch(const DropGeom &g, const Drop &d, const void *X, const void *R, void *Y, hipStream_t st)
{
    DropArgs a;
    a.wide = (int)((g.cols + 7) / 8);
    a.groups = g.rows * a.wide;
    a.cols = (int)g.cols;
    a.ld_x = g.ld_x;
    a.ld_r = g.ld_r;
    a.scale = g.alpha * d.scale;
    a.d = d;
    const long blocks = (a.groups + kThreads - 1) / kThreads, grid = blocks < 32768 ? blocks : 32768; // (16384 x 4096 with R: 77 us with 4096, 72 with 32768)
    a.step_rows = grid * kThreads / a.wide;
    a.step_cols = (int)(grid * kThreads % a.wide);
    auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3((unsigned)grid), dim3(kThreads), 0, st, a, (const T *)X, (const T *)R, (T *)Y); };
    if (g.cols % 8) go(R ? dropout_kernel<T, true, false> : dropout_kernel<T, false, false>);
    else go(R ? dropout_kernel<T, true, true> : dropout_kernel<T, false, true>);
    return hipGetLastError();
}

hipError_t launch_dropout(const DropGeom &g, const Drop &d, const void *X, const void *R, void *Y, hipStream_t st)
{
    return g.dtype == CAC_F32 ? launch<float>(g, d, X, R, Y, st) : launch<bf16_t>(g, d, X, R, Y, st);
}

} // namespace cac
