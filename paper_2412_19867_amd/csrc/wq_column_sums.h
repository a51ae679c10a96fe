// Sums over the rows of a matrix of partial sums, in 64 bits and in one order whatever the launch.
#pragma once

#include <hip/hip_runtime.h>

namespace {   // every including file has its own

// THREADS lanes: COLUMNS columns (64 or 16) x shares of the rows, eight rows of a share asked for at a time (one at a time each would wait for
// memory: 333 rows of 2560 8.2 us, so 5.1).  The sums of column c end up in the first COLUMNS lanes.
template <int COLUMNS, int THREADS>
__device__ __forceinline__ double column_sum(const float *part, int rows, long stride, long c, bool exists) {
    constexpr int SHARES = THREADS / COLUMNS;
    __shared__ double shares[THREADS / 64][COLUMNS];
    const int lane = threadIdx.x & 63, share = threadIdx.x / COLUMNS;
    double s = 0.0;
    if (exists)
        for (int r = share; r < rows; r += 8 * SHARES) {
            float v[8];
#pragma unroll
            for (int k = 0; k < 8; ++k) v[k] = part[(size_t)min(r + SHARES * k, rows - 1) * stride + c];
#pragma unroll
            for (int k = 0; k < 8; ++k) s += r + SHARES * k < rows ? (double)v[k] : 0.0;
        }
#pragma unroll
    for (int m = COLUMNS; m < 64; m <<= 1) s += __shfl_xor(s, m);
    if (lane < COLUMNS) shares[threadIdx.x >> 6][lane] = s;
    __syncthreads();
    s = 0.0;
    if (threadIdx.x < COLUMNS)
#pragma unroll
        for (int k = 0; k < THREADS / 64; ++k) s += shares[k][lane];
    return s;
}

}  // namespace
