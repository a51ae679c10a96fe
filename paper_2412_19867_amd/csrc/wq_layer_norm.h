// Statistics of a layer norm's rows, shared by the norm, its form that ends in codes, and its gradient.
#pragma once

#include "wq_quantize_piece.h"

namespace {   // every including file has its own

// Sums over a row of d = h - h[0] and of d^2 (and, for the gradient, of g = dy gamma and g d), in 64 bits: the shift takes away what rows far
// from zero would lose to the subtraction of the mean's square, so that one pass serves all of them; a constant row has variance 0.
template <int N>
__device__ __forceinline__ void wave_sums(double (&v)[N]) {
#pragma unroll
    for (int m = 32; m > 0; m >>= 1)
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] += __shfl_xor(v[i], m);
}

// 1 / sqrt(x), to the last places of 64 bits, from the hardware's estimate by two Newton steps.
__device__ __forceinline__ double rsqrt64(double x) {
    const double half = 0.5 * x;
    double y = __builtin_amdgcn_rsq(x);
    y = y * __builtin_fma(-half * y, y, 1.5);
    return y * __builtin_fma(-half * y, y, 1.5);
}

struct norm_stats {
    double mean;   // of h - h[0]
    double r;      // 1 / sqrt(var + eps)
};
__device__ __forceinline__ norm_stats stats_of(double sum, double squares, int C, double eps) {
    const double n = 1.0 / C, mean = sum * n, var = squares * n - mean * mean;
    return {mean, rsqrt64((var < 0.0 ? 0.0 : var) + eps)};   // (NaN stays)
}

// Elements c .. c + 7 of a row of `cols`, zero behind its end and (live false) everywhere; rows lie anywhere, elements are aligned to
// themselves.  Nothing branches on a lane: registers that one branch loads and another one fills would make each load wait for the
// one before (the gradient of 4096 rows of 8192 fp32 102 us so, 98 without).  A lane at the end reads the row's last eight
// and shifts them.  WHOLE: rows of whole eights.
template <typename T, bool WHOLE>
__device__ __forceinline__ void load8_row(const T *row, int c, int cols, bool live, float (&v)[8]) {
    if (!WHOLE && cols < 8) {
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = live && c + j < cols ? (float)row[c + j] : 0.0f;
        return;
    }
    const int at = min(c, cols - 8), shift = live ? c - at : 8;
    load8_anywhere<T>(row + at, v);
    if constexpr (!WHOLE) {
#pragma unroll
        for (int k = 1; k < 8; k <<= 1)
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] = shift & k ? (j + k < 8 ? v[j + k < 8 ? j + k : 0] : 0.0f) : v[j];
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = shift >= 8 ? 0.0f : v[j];
}
// Of a row's first `n` elements those from p on that exist.
template <typename T>
__device__ __forceinline__ void store8_some(T *p, int n, const float (&v)[8]) {
    if (n >= 8) {
        T t[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) t[j] = (T)v[j];
        __builtin_memcpy(p, t, sizeof t);
        return;
    }
#pragma unroll
    for (int j = 0; j < 8; ++j)
        if (j < n) p[j] = (T)v[j];
}

}  // namespace
