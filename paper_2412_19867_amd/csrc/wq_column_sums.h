// Sums over the rows of a matrix of partial sums, in 64 bits and in one order whatever the launch.
#pragma once

#include <hip/hip_runtime.h>

namespace {   // every including file has its own

// 1024 lanes: 64 columns x 16 shares of the rows, eight rows of a share asked for at a time (one at a time each would wait for memory:
// 333 rows of 2560 8.2 us, so 5.1).  The sums of column c end up in the first 64 lanes.
__device__ __forceinline__ double column_sum(const float *part, int rows, long stride, long c, bool exists) {
    __shared__ double shares[16][64];
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    double s = 0.0;
    if (exists)
        for (int r = w; r < rows; r += 128) {
            float v[8];
#pragma unroll
            for (int k = 0; k < 8; ++k) v[k] = part[(size_t)min(r + 16 * k, rows - 1) * stride + c];
#pragma unroll
            for (int k = 0; k < 8; ++k) s += r + 16 * k < rows ? (double)v[k] : 0.0;
        }
    shares[w][lane] = s;
    __syncthreads();
    s = 0.0;
    if (w == 0)
#pragma unroll
        for (int k = 0; k < 16; ++k) s += shares[k][lane];
    return s;
}

}  // namespace
