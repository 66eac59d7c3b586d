// Sums over the rows of a matrix of partial sums, in a fixed order: what the workgroups of a backward pass leave of the parameters' gradients.
#pragma once
#include "cawn_ops.hpp"

namespace cawn {
namespace ops {

// Sums of N values over the runs of a workgroup's threads, `each` threads a run: the first run has them then.  In halves: one after the other the 64 runs of
// a narrow matrix took longer than its reading (2 rows of 77 channels, the norm forward and backward: 31 us, so 12).  sh: N x THREADS.
template <int THREADS, int N> __device__ inline void over_runs(float (&v)[N], int runs, int each, float *sh)
{
    const int run = threadIdx.x / each;
    for (int half; runs > 1; runs = half) {
        half = (runs + 1) / 2;
        if (run >= half && run < runs) {
#pragma unroll
            for (int i = 0; i < N; ++i) sh[i * THREADS + threadIdx.x] = v[i];
        }
        __syncthreads();
        if (run + half < runs) {
#pragma unroll
            for (int i = 0; i < N; ++i) v[i] += sh[i * THREADS + threadIdx.x + half * each];
        }
    }
}

constexpr int SUM_COLS = 32, SUM_RUNS = 32;
constexpr long long SUM_BLOCKS = 1 << 14;       // workgroups at most (a launch counts its threads in 32 bits), which go round

// out(c) gives the place of column c's sum, or null.  A workgroup takes 32 columns; its 32 runs of threads take every 32nd row, and are
// added up in their order.  (With 16 and 8 columns a workgroup the backward passes that end in it are up to 6 and 17 % slower.)
template <typename Out> __device__ inline void sum_columns(const long long block, const float *part, const long long rows, const long long cols, const Out &out, const int accumulate)
{
    __shared__ float sh[SUM_RUNS][SUM_COLS + 1];
    const int col = threadIdx.x % SUM_COLS, run = threadIdx.x / SUM_COLS;
    const long long c = block * SUM_COLS + col;
    float v = 0.f;
    if (c < cols) {
        const float *p = part + c;
        long long r = run;
        for (; r + 3 * SUM_RUNS < rows; r += 4 * SUM_RUNS) {
            const float x0 = p[r * cols], x1 = p[(r + SUM_RUNS) * cols], x2 = p[(r + 2 * SUM_RUNS) * cols], x3 = p[(r + 3 * SUM_RUNS) * cols];
            v += (x0 + x1) + (x2 + x3);
        }
        for (; r < rows; r += SUM_RUNS) v += p[r * cols];
    }
    sh[run][col] = v;
    __syncthreads();
    if (run == 0 && c < cols) {
        float s = 0.f;
        for (int q = 0; q < SUM_RUNS; ++q) s += sh[q][col];
        float *at = out(c);
        if (at) *at = accumulate ? *at + s : s;
    }
}

template <typename Out> __global__ __launch_bounds__(SUM_COLS *SUM_RUNS) void column_sums(const float *part, const long long rows, const long long cols, const Out out,
                                                                                         const int accumulate)
{
    for (long long block = blockIdx.x; block * SUM_COLS < cols; block += gridDim.x) {
        if (block != blockIdx.x) __syncthreads();           // (the columns before have been added up)
        sum_columns(block, part, rows, cols, out, accumulate);
    }
}

template <typename Out> void launch_sums(const float *part, long long rows, long long cols, const Out &out, int accumulate, hipStream_t s)
{
    const long long blocks = ceil_div(cols, SUM_COLS) < SUM_BLOCKS ? ceil_div(cols, SUM_COLS) : SUM_BLOCKS;
    if (cols > 0) hipLaunchKernelGGL((column_sums<Out>), dim3((unsigned)blocks), dim3(SUM_COLS * SUM_RUNS), 0, s, part, rows, cols, out, accumulate);
}

} // namespace ops
} // namespace cawn
