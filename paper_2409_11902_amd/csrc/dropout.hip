// Dropout with its residual, Y = R + alpha * drop(X): a thread has groups of eight neighbours of a row, whose random bits it forms once.
// Bound by memory (dropout.h): X and R in and Y out, once.
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
    bool vector;
    float scale;
    Drop d;
};

template <typename T, bool RES> __global__ void __launch_bounds__(kThreads) dropout_kernel(const DropArgs a, const T *X, const T *R, T *Y)
{
    const DropKey key = drop_key(a.d);
    const long stride = (long)gridDim.x * kThreads;
    long g = (long)blockIdx.x * kThreads + threadIdx.x;
    long row = a.groups >> 32 ? g / a.wide : (long)((uint32_t)g / (uint32_t)a.wide);
    int col = (int)(g - row * a.wide);
    for (; g < a.groups; g += stride) {
        const int n = col * 8;
        Eight<T> x = read_eight(X + row * a.ld_x, n, a.cols, a.vector), r;
        if (RES) r = read_eight(R + row * a.ld_r, n, a.cols, a.vector);
        float v[8];
        x.get(v);
        drop_eight(key, a.d, (uint64_t)g, a.scale, v);
        if (RES) {
            float w[8];
            r.get(w);
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] += w[e];
        }
        write_eight(Y + row * a.cols, n, a.cols, a.vector, v);
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
    constexpr long kWhole = 16 / sizeof(T); // elements that start on 16 bytes
    DropArgs a;
    a.wide = (int)((g.cols + 7) / 8);
    a.groups = g.rows * a.wide;
    a.cols = (int)g.cols;
    a.ld_x = g.ld_x;
    a.ld_r = g.ld_r;
    a.vector = g.cols % 8 == 0 && g.ld_x % kWhole == 0 && (!R || g.ld_r % kWhole == 0);
    a.scale = g.alpha * d.scale;
    a.d = d;
    const long blocks = (a.groups + kThreads - 1) / kThreads, grid = blocks < 4096 ? blocks : 4096;
    a.step_rows = grid * kThreads / a.wide;
    a.step_cols = (int)(grid * kThreads % a.wide);
    if (R) hipLaunchKernelGGL((dropout_kernel<T, true>), dim3((unsigned)grid), dim3(kThreads), 0, st, a, (const T *)X, (const T *)R, (T *)Y);
    else hipLaunchKernelGGL((dropout_kernel<T, false>), dim3((unsigned)grid), dim3(kThreads), 0, st, a, (const T *)X, (const T *)nullptr, (T *)Y);
    return hipGetLastError();
}

hipError_t launch_dropout(const DropGeom &g, const Drop &d, const void *X, const void *R, void *Y, hipStream_t st)
{
    return g.dtype == CAC_F32 ? launch<float>(g, d, X, R, Y, st) : launch<bf16_t>(g, d, X, R, Y, st);
}

} // namespace cac
