// Sums over the rows of partial sums, in a fixed order.
#pragma once

#include "common.cuh"

namespace lf {

// Partial sums of the blocks of a kernel, joined channel by channel: 16 channels x 64 threads a block, each thread every 64th row, then
// the threads in pairs, always the same.
constexpr int kSumChannels = 16, kSumThreads = 1024;
static __global__ void __launch_bounds__(kSumThreads) column_sums_kernel(const float* partials, float* out, long long rows, int width, int C)
{
    constexpr int lanes = kSumThreads / kSumChannels;
    __shared__ float sums[lanes][kSumChannels];
    const int c = threadIdx.x % kSumChannels, l = threadIdx.x / kSumChannels, ch = blockIdx.x * kSumChannels + c;
    float a[8];
    pdl_wait();
    pdl_launch_dependents();
#pragma unroll
    for (int k = 0; k < 8; ++k) a[k] = 0.0f;
    for (long long r = l; r < rows; r += 8 * lanes)
#pragma unroll
        for (int k = 0; k < 8; ++k)
            if (r + k * lanes < rows) a[k] += partials[(r + k * lanes) * width + ch];
    sums[l][c] = ((a[0] + a[1]) + (a[2] + a[3])) + ((a[4] + a[5]) + (a[6] + a[7]));
    __syncthreads();
#pragma unroll
    for (int n = lanes / 2; n > 0; n /= 2) {
        if (l < n) sums[l][c] += sums[l + n][c];
        __syncthreads();
    }
    if (l == 0 && ch < C) out[ch] = sums[0][c];
}

}  // namespace lf
