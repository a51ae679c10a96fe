// Arguments of the quantized linear layer's product, and its epilogue: shared by the kernels of wq_linear*.hip.
#pragma once

#include "wq_device.h"
#include "wq_direct_plan.h"

struct wq_linear_args {
    const int8_t *xq, *Wq;
    const float *sx, *sW, *bias;
    const void *x;     // rows that the kernel quantizes itself, aligned to 16 bytes; null: xq and sx hold them
    const void *res;   // may be null; may be y itself
    void *y;
    long xs, rs, ys;   // row strides in elements
    int rows, P, Cin, Cout_pad, log2g;   // P: rows of the workspace's planes
    int outs;          // columns of y: Cout, or Cout / 2 with a gate
    int type, act, gated;
    bool wide;         // y and residual: every group of four columns lies in one aligned piece
};

// The tiled kernels (wq_linear_tile.h), 8-bit and 4-bit weights: workgroup tiles of 128 weight rows x 128 rows of x (`large`), or
// of 64 x 64 whose reduction 1, 2 or 4 teams of four waves share.
hipError_t wq_launch_linear_tile8(const wq_linear_args &a, int g, bool large, int teams, hipStream_t s);
hipError_t wq_launch_linear_tile4(const wq_linear_args &a, int g, bool large, int teams, hipStream_t s);
// Few rows: 16 nb rows of x to a workgroup, nb = 1 or 2 (wq_linear_rows.hip); with a.x the kernel quantizes them itself (nb = 1).
hipError_t wq_launch_linear_rows(const wq_linear_args &a, int g, int wbits, int nb, hipStream_t s);

namespace {   // every including file has its own

// 1 / (1 + e^-a) from e2 = -a log2(e): the hardware's exponential and reciprocal, each within a unit in the last place.
// e^-a beyond the range is infinite, its reciprocal zero.
__device__ __forceinline__ float logistic(float e2) { return __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(e2)); }

// The division, exponential and error function of the math library, correctly rounded or nearly, take 40 (silu) to 100 (gelu)
// instructions a value in place of 5 to 20: an eighth of the vector instructions of the product 4096 x 4096 -> 2 x 8192, g 128.
// G(x) = e^(x^2 / 2) erfc(x / sqrt 2) / 2 at x >= 0, so that Phi(-x) = e^(-x^2 / 2) G(x)
__device__ __forceinline__ float gelu_tail(float x) {
    // a polynomial in t = 1 / (1 + x / 4) that is 1/2 at x = 0: a fit by reweighted least squares of its relative error, 7e-8 up to x = 6,
    // 8e-7 at 10.  The negative tail keeps its digits so (a fit of one degree less, to the error of gelu itself, was 5e-7 off near 0 and
    // 2e-5 at -5; 2048x640->5120 g 64 W8 bf16 29.8 us with it, 30.5 so).
    const float t = __builtin_amdgcn_rcpf(__builtin_fmaf(0.25f, x, 1.0f));
    float G = -0.0996275544f;
    G = __builtin_fmaf(G, t, 0.380040318f);
    G = __builtin_fmaf(G, t, -0.343892276f);
    G = __builtin_fmaf(G, t, 0.364209324f);
    G = __builtin_fmaf(G, t, -0.0272250343f);
    G = __builtin_fmaf(G, t, 0.131000191f);
    G = __builtin_fmaf(G, t, 0.0952150896f);
    return __builtin_fmaf(G, t, 0.000279937405f);
}
__device__ __forceinline__ float gelu(float z) {
    // z Phi(z) = max(z, 0) - |z| Phi(-|z|)
    const float x = fabsf(z), G = gelu_tail(x);
    // (bounded from above: infinity times 0 would be NaN)
    const float b = fabsf(__builtin_elementwise_minimum(z, 0x1p60f));
    return __builtin_fmaf(-b, __builtin_amdgcn_exp2f(x * x * -0.721347520f) * G, fmaxf(z, 0.0f));
}

// N values at a time: one (uniform) choice for all of them.
template <int N>
__device__ __forceinline__ void activate(float (&z)[N], int act) {
    switch (act) {
        case WQ_ACT_RELU:
#pragma unroll
            for (int i = 0; i < N; ++i) z[i] = __builtin_elementwise_maximum(z[i], 0.0f);   // (the one that keeps a NaN)
            break;
        case WQ_ACT_SILU:
#pragma unroll
            for (int i = 0; i < N; ++i) z[i] *= logistic(z[i] * -1.44269504f);
            break;
        case WQ_ACT_GELU:
#pragma unroll
            for (int i = 0; i < N; ++i) z[i] = gelu(z[i]);
            break;
        case WQ_ACT_GELU_TANH:   // z (1 + tanh u) / 2 = z / (1 + e^-2u), u = sqrt(2 / pi) (z + 0.044715 z^3)
#pragma unroll
            for (int i = 0; i < N; ++i) z[i] *= logistic(z[i] * __builtin_fmaf(-0.102943240f, z[i] * z[i], -2.30220820f));
            break;
        default: break;
    }
}

typedef __bf16 v4bf __attribute__((ext_vector_type(4)));
typedef _Float16 v4h __attribute__((ext_vector_type(4)));

// Four adjacent elements from element `i` on.  `wide`: all four exist and lie in one aligned piece; otherwise `n` of
// them exist, each aligned to itself.
__device__ __forceinline__ v4f load_elems(const void *p, long i, int type, bool wide, int n) {
    v4f v = {0.f, 0.f, 0.f, 0.f};
    if (type == WQ_FP32) {
        const float *s = (const float *)p + i;
        if (wide) return *(const v4f *)s;
        for (int r = 0; r < 4; ++r)
            if (r < n) v[r] = s[r];
    } else if (type == WQ_BF16) {
        const __bf16 *s = (const __bf16 *)p + i;
        if (wide) return __builtin_convertvector(*(const v4bf *)s, v4f);
        for (int r = 0; r < 4; ++r)
            if (r < n) v[r] = (float)s[r];
    } else {
        const _Float16 *s = (const _Float16 *)p + i;
        if (wide) return __builtin_convertvector(*(const v4h *)s, v4f);
        for (int r = 0; r < 4; ++r)
            if (r < n) v[r] = (float)s[r];
    }
    return v;
}

__device__ __forceinline__ void store_elems(void *p, long i, int type, bool wide, int n, v4f v) {
    if (type == WQ_FP32) {
        float *d = (float *)p + i;
        if (wide) *(v4f *)d = v;
        else
            for (int r = 0; r < 4; ++r)
                if (r < n) d[r] = v[r];
    } else if (type == WQ_BF16) {
        __bf16 *d = (__bf16 *)p + i;
        const v4bf b = __builtin_convertvector(v, v4bf);
        if (wide) *(v4bf *)d = b;
        else
            for (int r = 0; r < 4; ++r)
                if (r < n) d[r] = b[r];
    } else {
        _Float16 *d = (_Float16 *)p + i;
        const v4h b = __builtin_convertvector(v, v4h);
        if (wide) *(v4h *)d = b;
        else
            for (int r = 0; r < 4; ++r)
                if (r < n) d[r] = b[r];
    }
}

// The epilogue of columns o .. o + 3 of rows p, p + row_step, .. (R of them), from the sums z (gated: and those of what the gate
// multiplies, up) with their bias, and the residual's values.
template <int R>
__device__ __forceinline__ void finish_columns(const wq_linear_args &a, long p, int row_step, int o, const v4f (&zs)[R],
                                               const v4f (&up)[R], const v4f (&res)[R]) {
    const int n = a.outs - o;
    float z[4 * R];
#pragma unroll
    for (int i = 0; i < 4 * R; ++i) z[i] = zs[i / 4][i % 4];
    activate(z, a.act);
#pragma unroll
    for (int r = 0; r < R; ++r) {
        v4f y = {z[4 * r], z[4 * r + 1], z[4 * r + 2], z[4 * r + 3]};
        if (a.gated) y *= up[r];
        if (a.res) y += res[r];
        if (p + r * row_step < a.rows) store_elems(a.y, (p + r * row_step) * a.ys + o, a.type, a.wide && n >= 4, n, y);
    }
}
__device__ __forceinline__ v4f residual_of(const wq_linear_args &a, long p, int o) {
    const int n = a.outs - o;
    return a.res && p < a.rows ? load_elems(a.res, p * a.rs + o, a.type, a.wide && n >= 4, n) : v4f{};
}

}  // namespace
